// gfx950 kernels of the optimizer step: AdamW over all tensors of a state,
// with moments in 32 or 8 bits and, if asked for, the chunk sums of what it
// wrote; the norm of the gradients; moments from one form to the other.
//
// All of them stream: an element's state is read and written once (28 bytes
// with bf16 gradients, 16 with 8-bit moments) for some 40 to 70 instructions, so
// HBM bounds them, at the 6.4-6.6 TB/s that a copy reaches (reads alone: 7.1);
// the 8-bit step comes near the vector units' bound as well (below).  A slot
// table says which tile of which tensor each workgroup takes, in address order,
// as in the restore's kernels.  What decides beyond that:
//
//   * The window.  A step reads three or four arrays and writes four, so the
//     memory that all workgroups touch at one time is seven windows, each as
//     wide as the tiles in flight.  With 8 workgroups of 256 threads and 2,048
//     elements on each compute unit the step of an 8B model's share (1.0e9
//     elements, bf16 gradients) ran at 6.3 TB/s in some allocations and 5.5 in
//     most, whatever the arrays' offsets to each other; the smaller the windows,
//     the smaller the gap.  One wave and 256 elements a workgroup and 10
//     workgroups a compute unit leave little of it: 4.32-4.48 ms in three
//     allocations, 6.3-6.5 TB/s (9: 4.38-4.50; 12: 4.33-4.53; 16: 4.45-4.63; no
//     bound: 4.73-4.77; 512 elements a wave, 8 to 32: 4.42-5.07; 128 threads, 5 a
//     compute unit: 4.39-4.60; 256 threads, 3: 4.35-4.59).  The number is set by
//     LDS that the launch asks for and nothing uses, as there is no other limit
//     short of the registers' (adamw.h).
//     With less work in flight the chain of dependent loads (slot, record,
//     hyperparameters, data) is what a tile waits for, so everything that does
//     not depend on the data is loaded before it, and computed behind it.
//     The other kernels have more instructions or fewer bytes a tile, which
//     takes more of them; their numbers (adamw.h) are from similar sweeps.
//   * Instructions, in 8 bits: hardware conversions from fp8 and to bf16, short
//     forms of root and quotient where the operands allow them, one scale a
//     wave (so that it is a scalar), codes rounded in place in the top bytes of
//     the words they are packed from: 83 -> 70 instructions an element, 2.92 ->
//     2.55-2.75 ms by allocation, 5.9-6.3 TB/s.  The vector units are then busy
//     for two thirds of it.
//   * Sums are folded by the wave that made them (wave_totals) and left 64 bytes
//     a tile for a second kernel: a step with them takes 4.5-4.9 ms by where the
//     arrays lie, where the step and a checksum of the state take 6.3 (8 bits:
//     2.8 and 3.8), in chunks of up to 16 MiB.  That kernel reads a chunk's parts
//     with one wave at most: from 64 MiB on it outlasts the checksum of a tensor
//     that few chunks hold (124M elements: 753 us where the two calls take 782,
//     8 bits 584 and 499; in chunks of 256 MiB 1,330 and 822, 768 and 536), and from
//     4 MiB on that of a small state (3.7M elements: 34 and 31, 23 and 23).
//   * No release and acquire between workgroups (finish_norm).
//
// The arithmetic is that of the header, operation by operation: no contraction
// to fused multiply-adds, sqrt and divisions correctly rounded.
#include <hip/hip_runtime.h>

#include "adamw.h"
#include "device.h"

#pragma clang fp contract(off)

namespace fr {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kDrop1 = 20, kDrop2 = 19;  // bits below a code of a first moment, of a root
constexpr int kLift = 112;               // codes at those bits stand for 2^-112 of their magnitudes

__device__ __forceinline__ float as_f(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t as_u(float f) { return __builtin_bit_cast(uint32_t, f); }

struct Tile {
  AdamwRec r;
  uint64_t e0;   // its first element
  uint32_t n;    // its elements
  uint32_t place;
};

// The tile of workgroup `block`: the slot of its own number or, with kRun > 1,
// one of kRun slots in order that the workgroups of one die take (workgroup b
// runs on die b mod 8), so that fewer lines of scales have parts in several L2s.
template <int T, int kRun>
__device__ __forceinline__ Tile tile_of(const AdamwWalk& w, const AdamwRec* recs, uint32_t block) {
  Tile t;
  uint64_t g = block;
  if constexpr (kRun > 1) {
    const uint32_t i = block % (8 * kRun), from = block - i;
    if (from + 8 * kRun <= uint32_t(w.n)) g = from + i % 8 * kRun + i / 8;
  }
  const uint64_t at = (g & 7) * w.stride + (g >> 3);
  const uint64_t slot = w.d[at];
  t.r = recs[slot >> 32];
  t.e0 = uint64_t(uint32_t(slot)) * T;
  // (in 32 bits: of `left < T ? left : T` in 64, which the callers' branch on a
  // whole tile compares again, clang 22 of ROCm 7.2.0 makes a vector comparison
  // and, behind the branch, a scalar select on the carry of an earlier sum)
  const uint32_t j = uint32_t(slot), whole = uint32_t(t.r.numel / T);
  t.n = j < whole ? uint32_t(T) : uint32_t(t.r.numel) % T;
  t.place = uint32_t(at);
  return t;
}

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

// ------------------------------------------------------------ 8-bit moments

// Four codes.  (Non-temporal, as everything that streams: with plain stores the
// conversion to 8 bits took 7 % longer.)
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p));
}
__device__ __forceinline__ void store_codes(uint32_t c, uint8_t* p) {
  __builtin_nontemporal_store(c, reinterpret_cast<uint32_t*>(p));
}

// Codes of elements i ... i + 3 and their block's scales (zeros behind the n > 0
// elements, by loads from the last place as in load4).
template <bool kFull>
__device__ __forceinline__ void load_block(const uint8_t* pm, const uint8_t* pv, const float* psm, const float* psv,
                                           uint32_t i, uint32_t n, uint32_t* cm, uint32_t* cv, float* sm, float* sv) {
  const uint32_t at = kFull || i < n ? i : (n - 1) & ~3u, b = at / FR_ADAMW_BLOCK;
  *cm = load_codes(pm + at);
  *cv = load_codes(pv + at);
  *sm = psm[b];
  *sv = psv[b];
  if (!kFull && i >= n) {
    *cm = *cv = 0;
    *sm = *sv = 0.0f;
  }
}

// The largest of a wave's 64 values, in all lanes (a scalar): four steps within
// rows of 16 lanes, two across them, by data-parallel primitives.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#define FR_DPP_MAX(ctrl)                                                              \
  {                                                                                   \
    const uint32_t y = __builtin_amdgcn_update_dpp(0u, x, ctrl, 0xF, 0xF, true);      \
    x = x > y ? x : y;                                                                \
  }
  FR_DPP_MAX(0x111)  // row_shr:1
  FR_DPP_MAX(0x112)
  FR_DPP_MAX(0x114)
  FR_DPP_MAX(0x118)
  FR_DPP_MAX(0x142)  // row_bcast:15
  FR_DPP_MAX(0x143)  // row_bcast:31
#undef FR_DPP_MAX
  return __builtin_amdgcn_readlane(x, 63);
}

// The larger magnitude, or NaN if one is (v_maximum3_f32).
__device__ __forceinline__ float larger(float a, float b) {
  return __builtin_elementwise_maximum(__builtin_fabsf(a), __builtin_fabsf(b));
}

// A wave's block: its scale, and the exponent that brings a value to where its
// code's bits are.  Scalars: every lane has the same.
struct Scale {
  float scale;
  int down;
  bool bad;  // stands for NaN
};
__device__ __forceinline__ Scale scale_of(float largest) {
  const uint32_t top = wave_max(as_u(largest) & 0x7FFFFFFFu);
  const int e = (int(top - 1) >> 23) + 1;  // of the smallest power of two not below it
  Scale s;
  s.bad = e >= 254;
  s.scale = e < 28 ? 0.0f : s.bad ? as_f(0x7FC00000u) : as_f(uint32_t(e) << 23);
  s.down = e < 28 ? -1000 : 127 - e - kLift;  // (to zeros)
  return s;
}

// Four first moments from their codes: as OCP e4m3 numbers the codes stand for
// 2^8 times what they do here.
__device__ __forceinline__ f32x4 decode1(uint32_t c, float scale) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
  const float k = scale * 0x1p-8f;
  return f32x4{a[0] * k, a[1] * k, b[0] * k, b[1] * k};
}
// Four second moments from the codes of their roots.  `scale` is the wave's.
__device__ __forceinline__ f32x4 decode2(uint32_t c, float scale) {
  constexpr uint32_t kBits = 255u << kDrop2;
  const uint32_t e = as_u(scale) >> 23;
  const int up = e ? int(e) - 127 + kLift : -1000;           // (a scale of 0: zeros)
  const uint32_t bad = e == 255 ? as_u(scale) : 0u;           // (NaN, whatever the codes)
  f32x4 v;
#pragma unroll
  for (int j = 0; j < 4; j++) {
    const int shift = 8 * j - kDrop2;
    const uint32_t u = ((shift < 0 ? c << -shift : c >> shift) & kBits) | bad;
    const float r = __builtin_amdgcn_ldexpf(as_f(u), up);
    v[j] = r * r;
  }
  return v;
}

// What is added to four elements' patterns before the bits below their codes
// are dropped.  The low bits of the counter of the first are 0, so that the
// products of the four differ by constants.
struct Noise {
  uint32_t m[4], r[4];
};
__device__ __forceinline__ Noise noise4(uint64_t counter, uint32_t seed) {
  Noise x;
  if (seed == 0) {
#pragma unroll
    for (int j = 0; j < 4; j++) {
      x.m[j] = 1u << (kDrop1 - 1);
      x.r[j] = 1u << (kDrop2 - 1);
    }
    return x;
  }
  constexpr uint32_t k1 = 0x9E3779B9u;
  const uint32_t high = uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(counter >> 32))) * 0x85157AF5u;
  const uint32_t p = ((uint32_t(counter) ^ high) & ~3u) * k1;
#pragma unroll
  for (uint32_t j = 0; j < 4; j++) {
    // (kept a scalar, so that four products do not become of one)
    uint32_t h = p + __builtin_amdgcn_readfirstlane(((high & 3u) ^ j) * k1 + seed);
    h ^= h >> 16;
    h *= 0xB504F333u;
    h ^= h >> 15;
    h *= 0x93CD3A2Du;
    h ^= h >> 16;
    x.m[j] = h >> 12;
    x.r[j] = h & 0x7FFFFu;
  }
  return x;
}

// The top bytes of four words.
__device__ __forceinline__ uint32_t pack_top(const uint32_t (&x)[4]) {
  return __builtin_amdgcn_perm(x[1], x[0], 0x0C0C0703u) | __builtin_amdgcn_perm(x[3], x[2], 0x07030C0Cu);
}

// Codes of four first moments and four roots of second ones, which with those
// of the wave's other lanes make up a block; the block's scales.
__device__ __forceinline__ void encode4(const f32x4& m, const f32x4& r, uint64_t counter, uint32_t seed,
                                        uint32_t* cm, uint32_t* cr, float* sm, float* sr) {
  const Scale xm = scale_of(larger(larger(m[0], m[1]), larger(m[2], m[3])));
  const Scale xr = scale_of(larger(larger(r[0], r[1]), larger(r[2], r[3])));
  const Noise z = noise4(counter, seed);
  uint32_t a[4], b[4];  // codes in the top bytes
#pragma unroll
  for (int j = 0; j < 4; j++) {
    const uint32_t u = (as_u(__builtin_amdgcn_ldexpf(m[j], xm.down)) + z.m[j]) << (24 - kDrop1);
    a[j] = (u & 0x7FFFFFFFu) | (as_u(m[j]) & 0x80000000u);
    b[j] = (as_u(__builtin_amdgcn_ldexpf(r[j], xr.down)) + z.r[j]) << (24 - kDrop2);
  }
  *cm = pack_top(a) & (xm.bad ? 0x80808080u : ~0u);
  *cr = pack_top(b) & (xr.bad ? 0u : ~0u);
  *sm = xm.scale;
  *sr = xr.scale;
}

// Four fp32 patterns to bf16, two a word: v_cvt_pk_bf16_f32 rounds every
// pattern as rne_bf16 does, NaNs included.
__device__ __forceinline__ u32x2 to_bf16(const f32x4& x) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(x.xy, bf16x2)),
               __builtin_bit_cast(uint32_t, __builtin_convertvector(x.zw, bf16x2))};
}

// ------------------------------------------------ square roots and quotients

// Square roots and divisions in their general form take 13 and 11 instructions,
// a third of them for operands near the ends of the range.  Where all of a
// wave's operands are well inside it, these give the same correctly rounded
// results by an approximation and Newton steps with exact residuals (fused
// multiply-adds), as P. Markstein, "Computation of elementary functions on the
// IBM RISC System/6000 processor" (1990), shows: a quotient that is within one
// unit of its last place, corrected by its residual times a correctly rounded
// reciprocal, is correctly rounded.  (m * y may be off by up to one and a half
// where m's mantissa is the smaller one: the 2.2e8 quotients of 24-bit numbers
// nearest to a border, over all divisors, come out right all the same, and with
// a reciprocal that is one unit off 5e6 of them do not.)  The tests compare
// these, and on the device every root of three pairs of binades, the ranges'
// ends among them, and its quotients with the numerators hardest to round.
__device__ __forceinline__ float root_inside(float v) {  // 2^-96 <= v <= 2^126 (NaN of a negative one)
  const float y = __builtin_amdgcn_rsqf(v), g = v * y;
  return __builtin_fmaf(__builtin_fmaf(-g, g, v), 0.5f * y, g);
}
__device__ __forceinline__ float quotient_inside(float m, float d) {  // 2^-80 <= |m| <= 2^60, 2^-60 <= d <= 2^40
  const float y0 = __builtin_amdgcn_rcpf(d);
  const float y = __builtin_fmaf(__builtin_fmaf(-d, y0, 1.0f), y0, y0), q = m * y;
  return __builtin_fmaf(__builtin_fmaf(-d, q, m), y, q);
}
// Whether the magnitudes of all of a wave's values lie in [lo, hi]; no NaN does.
__device__ __forceinline__ bool inside(const f32x4& x, float lo, float hi) {
  const auto least = [](float a, float b) { return __builtin_elementwise_minimum(__builtin_fabsf(a), __builtin_fabsf(b)); };
  const float a = least(least(x[0], x[1]), least(x[2], x[3])), b = larger(larger(x[0], x[1]), larger(x[2], x[3]));
  return __all(a >= lo && b <= hi);
}
__device__ __forceinline__ f32x4 roots(const f32x4& v) {
  f32x4 r;
  if (inside(v, 0x1p-96f, 0x1p126f)) {
#pragma unroll
    for (int j = 0; j < 4; j++) r[j] = root_inside(v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; j++) r[j] = __builtin_sqrtf(v[j]);
  }
  return r;
}

// --------------------------------------------------------------------- step

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

// A value that is the same in all of a wave's lanes that hold one (lane 0 does).
__device__ __forceinline__ float wave_scalar(float x) { return as_f(__builtin_amdgcn_readfirstlane(as_u(x))); }

// Where a tile's arrays are.
struct StepCtx {
  uint8_t *pw, *pp, *pm, *pv;
  float *psm, *psv;
  const uint8_t* pg;
  uint32_t n;
  uint64_t counter;
  fr_adamw_hyper hyper;  // its group's
  fr_grad_stats stats;
  uint32_t word4, word2, word1;  // first word of the tile in its chunks, by bytes an element
};

// The constants of a step, each with the header's roundings.
struct StepConsts {
  float gs, beta1, a1, beta2, a2, rb2, eps, keep, lr;
  uint32_t seed;
  bool skip;
  bool inside;  // with |v| in [2^-96, 2^60] the divisor is in [2^-60, 2^40], or NaN (of a negative v)
};
__device__ __forceinline__ StepConsts consts_of(const fr_adamw_hyper& h, const fr_grad_stats& g) {
  StepConsts c;
  c.skip = g.nonfinite != 0;
  c.gs = g.scale;
  c.beta1 = h.beta1;
  c.a1 = 1.0f - h.beta1;
  c.beta2 = h.beta2;
  c.a2 = 1.0f - h.beta2;
  c.rb2 = 1.0f / __builtin_sqrtf(h.bias2);
  c.eps = h.eps;
  c.keep = 1.0f - h.lr * h.weight_decay;
  c.lr = h.lr / h.bias1;
  c.seed = h.seed;
  c.inside = c.rb2 >= 0x1p-10f && c.rb2 <= 0x1p8f && c.eps >= 0.0f && c.eps <= 0x1p39f;
  return c;
}

// One tile.  kFull: it is whole, so that nothing is predicated; kGrad32: fp32
// gradients.  All loads are issued before anything is waited for, the
// constants among it.
template <bool kEight, bool kSums, bool kFull, bool kGrad32, int B, int U>
__device__ __forceinline__ void step_tile(const StepCtx& t, u64 (&s)[kSummed], u64 (&ws)[kSummed]) {
  const uint32_t n = kFull ? B * U * 4 : t.n;
  u32x4 uw[U], um[U], uv[U], ug[U];
  uint32_t cm[U] = {}, cv[U] = {};
  float sm[U] = {}, sv[U] = {};
#pragma unroll
  for (int q = 0; q < U; q++) {
    const uint32_t i = (q * B + threadIdx.x) * 4;
    uw[q] = load4<kFull>(t.pw, i, n);
    if constexpr (kEight) {
      load_block<kFull>(t.pm, t.pv, t.psm, t.psv, i, n, &cm[q], &cv[q], &sm[q], &sv[q]);
    } else {
      um[q] = load4<kFull>(t.pm, i, n);
      uv[q] = load4<kFull>(t.pv, i, n);
    }
    ug[q] = kGrad32 ? load4<kFull>(t.pg, i, n) : load4h<kFull>(t.pg, i, n);
  }
  const StepConsts k = consts_of(t.hyper, t.stats);
  if (k.skip && !kSums) return;
#pragma unroll
  for (int q = 0; q < U; q++) {
    const uint32_t i = (q * B + threadIdx.x) * 4, b = i / FR_ADAMW_BLOCK;  // the wave's block
    f32x4 m, v;
    u32x2 up = {0, 0};
    if constexpr (kEight) {
      m = decode1(cm[q], wave_scalar(sm[q]));
      v = decode2(cv[q], wave_scalar(sv[q]));
    } else {
      m = __builtin_bit_cast(f32x4, um[q]);
      v = __builtin_bit_cast(f32x4, uv[q]);
    }
    if (!k.skip) {
      const f32x4 g = __builtin_bit_cast(f32x4, kGrad32 ? ug[q] : widen(ug[q]));
      f32x4 w = __builtin_bit_cast(f32x4, uw[q]), root;
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const float x = g[j] * k.gs;
        m[j] = m[j] * k.beta1 + x * k.a1;
        v[j] = v[j] * k.beta2 + (x * x) * k.a2;
      }
      f32x4 quotient;
      if (k.inside && inside(m, 0x1p-80f, 0x1p60f) && inside(v, 0x1p-96f, 0x1p60f)) {
#pragma unroll
        for (int j = 0; j < 4; j++) {
          root[j] = root_inside(v[j]);
          quotient[j] = quotient_inside(m[j], root[j] * k.rb2 + k.eps);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; j++) {
          root[j] = __builtin_sqrtf(v[j]);
          quotient[j] = m[j] / (root[j] * k.rb2 + k.eps);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; j++) {
        w[j] = w[j] * k.keep - quotient[j] * k.lr;
        if (!kFull && i + j >= n) m[j] = v[j] = w[j] = root[j] = 0.0f;  // eps may be 0
      }
      uw[q] = __builtin_bit_cast(u32x4, w);
      up = to_bf16(w);
      store4<kFull>(t.pw, uw[q], i, n);
      if (t.pp) store4h<kFull>(t.pp, up, i, n);
      if constexpr (kEight) {
        encode4(m, root, t.counter + i, k.seed, &cm[q], &cv[q], &sm[q], &sv[q]);
        if (kFull || i < n) {
          store_codes(cm[q], t.pm + i);
          store_codes(cv[q], t.pv + i);
          if (threadIdx.x % 64 == 0) {
            t.psm[b] = sm[q];
            t.psv[b] = sv[q];
          }
        }
      } else {
        um[q] = __builtin_bit_cast(u32x4, m);
        uv[q] = __builtin_bit_cast(u32x4, v);
        store4<kFull>(t.pm, um[q], i, n);
        store4<kFull>(t.pv, uv[q], i, n);
      }
    } else if (t.pp) {
      const u32x4 x = widen(load4h<kFull>(t.pp, i, n));
      up = u32x2{x.x >> 16 | x.y, x.z >> 16 | x.w};
    }
    if constexpr (kSums) {
      if (t.pp) acc2(up, t.word2 + i / 2, s[kParam], ws[kParam]);
      acc4(uw[q], t.word4 + i, s[kMaster], ws[kMaster]);
      if constexpr (kEight) {
        const u64 i1 = t.word1 + i / 4 + 1;
        s[kMom1] += cm[q];
        ws[kMom1] += i1 * cm[q];
        s[kMom2] += cv[q];
        ws[kMom2] += i1 * cv[q];
      } else {
        acc4(um[q], t.word4 + i, s[kMom1], ws[kMom1]);
        acc4(uv[q], t.word4 + i, s[kMom2], ws[kMom2]);
      }
    }
  }
}

template <bool kEight, bool kSums, int B, int U, int kRun>
__global__ __launch_bounds__(B) void k_adamw(const AdamwRec* __restrict__ recs, AdamwWalk walk,
                                             uint8_t* __restrict__ state, const uint8_t* __restrict__ grads,
                                             const fr_adamw_hyper* __restrict__ hyper,
                                             const fr_grad_stats* __restrict__ stats, uint64_t C,
                                             fr_chunk_sum* __restrict__ parts) {
  const Tile t = tile_of<B * U * 4, kRun>(walk, recs, blockIdx.x);
  StepCtx c;
  c.n = t.n;
  c.hyper = hyper[t.r.group];
  c.stats = *stats;
  c.pw = state + t.r.at[kMaster] + 4 * t.e0;
  c.pp = t.r.at[kParam] == kNone ? nullptr : state + t.r.at[kParam] + 2 * t.e0;
  c.pm = state + t.r.at[kMom1] + (kEight ? 1 : 4) * t.e0;
  c.pv = state + t.r.at[kMom2] + (kEight ? 1 : 4) * t.e0;
  c.psm = kEight ? reinterpret_cast<float*>(state + t.r.at[kScale1]) + t.e0 / FR_ADAMW_BLOCK : nullptr;
  c.psv = kEight ? reinterpret_cast<float*>(state + t.r.at[kScale2]) + t.e0 / FR_ADAMW_BLOCK : nullptr;
  c.pg = grads + t.r.grad + (t.r.grad_f32 ? 4 : 2) * t.e0;
  c.counter = t.r.counter + t.e0;

  if (kSums) {
    const uint64_t mask = C - 1;
    c.word4 = uint32_t(4 * t.e0 & mask) / 4;
    c.word2 = uint32_t(2 * t.e0 & mask) / 4;
    c.word1 = uint32_t(t.e0 & mask) / 4;
  }

  u64 s[kSummed] = {}, ws[kSummed] = {};
  if (t.n == B * U * 4) {
    if (t.r.grad_f32) step_tile<kEight, kSums, true, true, B, U>(c, s, ws);
    else step_tile<kEight, kSums, true, false, B, U>(c, s, ws);
  } else {
    if (t.r.grad_f32) step_tile<kEight, kSums, false, true, B, U>(c, s, ws);
    else step_tile<kEight, kSums, false, false, B, U>(c, s, ws);
  }
  if constexpr (kSums) {
    static_assert(B == 64, "a wave");
    u64 x[8];
#pragma unroll
    for (int k = 0; k < 4; k++) {
      x[2 * k] = s[k];
      x[2 * k + 1] = ws[k];
    }
    const u64 total = wave_totals(x);
    const uint32_t v = threadIdx.x / 8;
    if (threadIdx.x % 8 == 0)
      reinterpret_cast<u64*>(parts + (uint64_t(v / 2) * 8 * walk.stride + t.place))[v % 2] = total;
  }
}

// The sums of chunks.  The first n_scales workgroups read a chunk of scales
// each; the others take what the tiles of a chunk left, L lanes a chunk and four
// loads of each in flight (past the end the last one again, not counted).  Places
// are kept array by array, so that what one chunk needs is contiguous.  A wave a
// chunk costs an 8B model's share in chunks of 64 KiB, 215,000 of them, 97 us
// where 16 lanes take 59; a chunk of 512 tiles wants the wave (a state of 3.7M
// elements, chunks of 256 KiB, step and sums: 26.1 us with 16 lanes, 23.6 with 64).
template <uint32_t L>
__global__ __launch_bounds__(256) void k_adamw_fold(const AdamwFold* folds, uint32_t n_folds,
                                                    const AdamwScales* scales, uint32_t n_scales, uint64_t stride,
                                                    const fr_chunk_sum* parts, const uint8_t* state,
                                                    fr_chunk_sum* sums) {
  u64 s = 0, ws = 0;
  if (blockIdx.x < n_scales) {
    const AdamwScales d = scales[blockIdx.x];
    const u32x4* const p = reinterpret_cast<const u32x4*>(state + d.at);
#pragma unroll 4
    for (uint32_t i = threadIdx.x; i < d.words / 4; i += 256) acc4(p[i], 4 * i, s, ws);
    const uint32_t last = d.words / 4 * 4 + threadIdx.x;
    if (last < d.words) {
      const uint32_t w = reinterpret_cast<const uint32_t*>(p)[last];
      s += w;
      ws += u64(last + 1) * w;
    }
    __shared__ u64 part[8];
#pragma unroll
    for (int x = 32; x; x >>= 1) {
      s += __shfl_xor(s, x);
      ws += __shfl_xor(ws, x);
    }
    if (threadIdx.x % 64 == 0) {
      part[threadIdx.x / 64] = s;
      part[4 + threadIdx.x / 64] = ws;
    }
    __syncthreads();
    if (threadIdx.x == 0)
      sums[d.chunk] = fr_chunk_sum{part[0] + part[1] + part[2] + part[3], part[4] + part[5] + part[6] + part[7]};
    return;
  }
  const uint32_t f = ((blockIdx.x - n_scales) * 256 + threadIdx.x) / L, lane = threadIdx.x % L;
  AdamwFold d = {};
  if (f < n_folds) {
    d = folds[f];
    const fr_chunk_sum* const p = parts + uint64_t(d.kind) * 8 * stride;
    constexpr uint32_t kLoads = 4;
    for (uint32_t j = lane; j < d.n; j += kLoads * L) {
      fr_chunk_sum x[kLoads];
#pragma unroll
      for (uint32_t k = 0; k < kLoads; k++) {
        const uint64_t g = uint64_t(d.slot) + (j + k * L < d.n ? j + k * L : d.n - 1);
        x[k] = p[(g & 7) * stride + (g >> 3)];
      }
#pragma unroll
      for (uint32_t k = 0; k < kLoads; k++) {
        s += j + k * L < d.n ? x[k].sum : 0;
        ws += j + k * L < d.n ? x[k].wsum : 0;
      }
    }
  }
#pragma unroll
  for (int x = L / 2; x; x >>= 1) {
    s += __shfl_xor(s, x);
    ws += __shfl_xor(ws, x);
  }
  if (f < n_folds && lane == 0) sums[d.chunk] = fr_chunk_sum{s, ws};
}

// --------------------------------------------------------------------- norm

// (A norm past fp32's range, of gradients that are finite, still has a scale: a
// quotient of infinity would step with gradients of zero.)
__device__ __forceinline__ void set_stats(double sum_sq, float max_norm, fr_grad_stats* out) {
  const bool fine = __builtin_isfinite(sum_sq);
  const double root = __builtin_sqrt(sum_sq);
  const float norm = float(root);
  const float clip = __builtin_isfinite(norm) ? max_norm / norm : float(double(max_norm) / root);
  out->sum_sq = sum_sq;
  out->norm = norm;
  out->scale = !fine ? 0.0f : norm > max_norm ? clip : 1.0f;
  out->nonfinite = fine ? 0 : 1;
}

__device__ __forceinline__ double block_sum(double x) {
  __shared__ double part[4];
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = x;
  __syncthreads();
  x = part[0] + part[1] + part[2] + part[3];
  __syncthreads();
  return x;
}

// The sum of the squares of a thread's share of one tile.  kFull: the tile is
// whole, and all its loads are in flight before the first is used.
template <bool kFull, bool kGrad32>
__device__ __forceinline__ double squares(const uint8_t* p, uint32_t n) {
  double sum = 0;
  if constexpr (kFull) {
    constexpr int V = kNormBytes / (256 * 16);
    u32x4 x[V];
#pragma unroll
    for (int q = 0; q < V; q++) x[q] = ld_nt(reinterpret_cast<const u32x4*>(p) + q * 256 + threadIdx.x);
#pragma unroll
    for (int q = 0; q < V; q++)
#pragma unroll
      for (int j = 0; j < 4; j++) {
        if (kGrad32) {
          const double a = as_f(x[q][j]);
          sum += a * a;
        } else {
          const double a = as_f(x[q][j] << 16), b = as_f(x[q][j] & 0xFFFF0000u);
          sum += a * a;
          sum += b * b;
        }
      }
  } else {
    for (uint32_t i = threadIdx.x * 4; i < n; i += 256 * 4) {
      const f32x4 x = __builtin_bit_cast(f32x4, kGrad32 ? load4<false>(p, i, n) : widen(load4h<false>(p, i, n)));
      for (int j = 0; j < 4; j++) sum += double(x[j]) * double(x[j]);
    }
  }
  return sum;
}

// Adds one arrival of `of` at a line; whether it was the last one, for which
// the line is left at zero.
__device__ __forceinline__ bool arrive_last(uint32_t* lines, uint32_t line, uint32_t of) {
  uint32_t* p = lines + line * (kNormLine / 4);
  if (__hip_atomic_fetch_add(p, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != of - 1) return false;
  __hip_atomic_store(p, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return true;
}

// The end of a workgroup's part `sum` (thread 0's) of a norm: it is left at
// parts[blockIdx.x]; whoever arrives last adds up all, each thread and the
// whole in an order of their own, whoever it is.  A part is exchanged, not
// stored, and its return waited for before the arrival is added: it is then
// where every other workgroup's atomic loads find it, without the release
// and acquire that write back and invalidate a whole L2 each (1,800 of them
// took 35 us).
__device__ __forceinline__ void finish_norm(double sum, double* parts, uint32_t* arrived, float max_norm,
                                            fr_grad_stats* stats) {
  __shared__ bool last;
  if (threadIdx.x == 0) {
    const unsigned long long before = __hip_atomic_exchange(
        reinterpret_cast<unsigned long long*>(parts + blockIdx.x), __builtin_bit_cast(unsigned long long, sum),
        __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // (unused, it would be compiled to the form without a return)
    asm volatile("s_waitcnt vmcnt(0)" ::"v"(before) : "memory");
    const uint32_t lines = (gridDim.x + kNormPerLine - 1) / kNormPerLine, line = blockIdx.x % lines;
    last = gridDim.x <= kNormOneLine
               ? arrive_last(arrived, 0, gridDim.x)
               : arrive_last(arrived, 1 + line, (gridDim.x - line + lines - 1) / lines) && arrive_last(arrived, 0, lines);
  }
  __syncthreads();
  if (!last) return;
  sum = 0;
  for (uint32_t i = threadIdx.x; i < gridDim.x; i += 256)
    sum += __hip_atomic_load(parts + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  sum = block_sum(sum);
  if (threadIdx.x == 0) set_stats(sum, max_norm, stats);
}

// One tile a workgroup.  kOne: the only launch of the norm; else its part goes
// to its place for k_norm_fold.
template <bool kOne>
__global__ __launch_bounds__(256) void k_norm(const AdamwRec* recs, AdamwWalk walk, const uint8_t* grads,
                                              float max_norm, fr_grad_stats* stats, double* parts,
                                              uint32_t* arrived) {
  double sum = 0;
  const uint32_t g = blockIdx.x, at = (g & 7) * uint32_t(walk.stride) + (g >> 3);
  if (!kOne || walk.n) {  // (no tiles: one workgroup, of nothing)
    const uint64_t slot = walk.d[at];
    const AdamwRec& r = recs[slot >> 32];
    const uint8_t* const p = grads + r.grad + uint64_t(uint32_t(slot)) * kNormBytes;
    const bool f32 = r.grad_f32 != 0;
    const uint32_t T = kNormBytes / (f32 ? 4 : 2), whole = uint32_t(r.numel / T);
    if (uint32_t(slot) < whole) sum = f32 ? squares<true, true>(p, T) : squares<true, false>(p, T);
    else sum = f32 ? squares<false, true>(p, uint32_t(r.numel) % T) : squares<false, false>(p, uint32_t(r.numel) % T);
  }
  sum = block_sum(sum);
  if constexpr (kOne) finish_norm(sum, parts, arrived, max_norm, stats);
  else if (threadIdx.x == 0) parts[at] = sum;
}

// The sum of the places' parts: each workgroup adds a run of them up.
__global__ __launch_bounds__(256) void k_norm_fold(uint64_t stride, uint64_t n, double* parts, double* parts2,
                                                   float max_norm, fr_grad_stats* stats, uint32_t* arrived) {
  const uint32_t places = 8 * uint32_t(stride), run = (places + gridDim.x - 1) / gridDim.x;
  const uint32_t first = blockIdx.x * run, end = first + run < places ? first + run : places;
  double sum = 0;
  for (uint32_t i = first + threadIdx.x; i < end; i += 256) {
    const uint32_t x = i / uint32_t(stride);
    if ((i - x * uint32_t(stride)) * 8 + x < uint32_t(n)) sum += parts[i];  // the others are no workgroup's
  }
  sum = block_sum(sum);
  finish_norm(sum, parts2, arrived, max_norm, stats);
}

__global__ void k_scale(float max_norm, fr_grad_stats* stats) { set_stats(stats->sum_sq, max_norm, stats); }

// ------------------------------------------------------------------ convert

struct ConvertCtx {
  const uint8_t *qm, *qv;
  const float *qsm, *qsv;
  uint8_t *pm, *pv;
  float *psm, *psv;
  uint32_t n, seed;
  uint64_t counter;
};

// One tile; k8From, k8To: the forms.  All loads are issued before the first is
// used.
template <bool k8From, bool k8To, bool kFull, int B, int U>
__device__ __forceinline__ void convert_tile(const ConvertCtx& t) {
  const uint32_t n = kFull ? B * U * 4 : t.n;
  u32x4 um[U], uv[U];
  uint32_t cm[U] = {}, cv[U] = {};
  float sm[U] = {}, sv[U] = {};
#pragma unroll
  for (int q = 0; q < U; q++) {
    const uint32_t i = (q * B + threadIdx.x) * 4;
    if constexpr (k8From) {
      load_block<kFull>(t.qm, t.qv, t.qsm, t.qsv, i, n, &cm[q], &cv[q], &sm[q], &sv[q]);
    } else {
      um[q] = load4<kFull>(t.qm, i, n);
      uv[q] = load4<kFull>(t.qv, i, n);
    }
  }
#pragma unroll
  for (int q = 0; q < U; q++) {
    const uint32_t i = (q * B + threadIdx.x) * 4, b = i / FR_ADAMW_BLOCK;
    if constexpr (k8From && !k8To) {
      um[q] = __builtin_bit_cast(u32x4, decode1(cm[q], wave_scalar(sm[q])));
      uv[q] = __builtin_bit_cast(u32x4, decode2(cv[q], wave_scalar(sv[q])));
    }
    if constexpr (!k8From && k8To) {
      const f32x4 r = roots(__builtin_bit_cast(f32x4, uv[q]));
      encode4(__builtin_bit_cast(f32x4, um[q]), r, t.counter + i, t.seed, &cm[q], &cv[q], &sm[q], &sv[q]);
    }
    if constexpr (k8To) {
      if (kFull || i < n) {
        store_codes(cm[q], t.pm + i);
        store_codes(cv[q], t.pv + i);
        if (threadIdx.x % 64 == 0) {
          t.psm[b] = sm[q];
          t.psv[b] = sv[q];
        }
      }
    } else {
      store4<kFull>(t.pm, um[q], i, n);
      store4<kFull>(t.pv, uv[q], i, n);
    }
  }
}

template <bool k8To, int B, int U, int kRun>
__global__ __launch_bounds__(B) void k_convert(const AdamwRec* from_recs, const AdamwRec* to_recs, AdamwWalk walk,
                                               const uint8_t* from, uint8_t* to, uint32_t seed) {
  const Tile t = tile_of<B * U * 4, kRun>(walk, to_recs, blockIdx.x);
  const AdamwRec f = from_recs[walk.d[t.place] >> 32];
  const bool f8 = f.at[kScale1] != kNone;
  const uint64_t b0 = t.e0 / FR_ADAMW_BLOCK;
  ConvertCtx c;
  c.qm = from + f.at[kMom1] + (f8 ? 1 : 4) * t.e0;
  c.qv = from + f.at[kMom2] + (f8 ? 1 : 4) * t.e0;
  c.qsm = f8 ? reinterpret_cast<const float*>(from + f.at[kScale1]) + b0 : nullptr;
  c.qsv = f8 ? reinterpret_cast<const float*>(from + f.at[kScale2]) + b0 : nullptr;
  c.pm = to + t.r.at[kMom1] + (k8To ? 1 : 4) * t.e0;
  c.pv = to + t.r.at[kMom2] + (k8To ? 1 : 4) * t.e0;
  c.psm = k8To ? reinterpret_cast<float*>(to + t.r.at[kScale1]) + b0 : nullptr;
  c.psv = k8To ? reinterpret_cast<float*>(to + t.r.at[kScale2]) + b0 : nullptr;
  c.n = t.n;
  c.seed = seed;
  c.counter = t.r.counter + t.e0;
  if (t.n == B * U * 4) {
    if (f8) convert_tile<true, k8To, true, B, U>(c);
    else convert_tile<false, k8To, true, B, U>(c);
  } else {
    if (f8) convert_tile<true, k8To, false, B, U>(c);
    else convert_tile<false, k8To, false, B, U>(c);
  }
}

template <bool kEight, bool kSums>
int step(const AdamwStepArgs& a, hipStream_t st) {
  constexpr AdamwShape s = kSums ? kSumShape[kEight] : kStepShape[kEight];
  hipLaunchKernelGGL((k_adamw<kEight, kSums, s.B, s.U, s.run>), dim3(uint32_t(a.walk.n)), dim3(s.B), s.lds, st, a.recs,
                     a.walk, static_cast<uint8_t*>(a.state), static_cast<const uint8_t*>(a.grads), a.hyper, a.stats,
                     a.C, a.parts);
  const int e = int(hipGetLastError());
  if (e != 0 || !kSums || a.n_folds == 0) return e;
  // tiles of the longest chunks that are fed by tiles: parameters', or codes'
  const uint64_t tiles = a.C / (kEight ? 1 : 2) / s.tile();
  const auto fold = [&](auto kernel, uint32_t lanes) {
    const uint32_t per = 256 / lanes;
    hipLaunchKernelGGL(kernel, dim3(a.n_scales + (a.n_folds + per - 1) / per), dim3(256), 0, st, a.folds, a.n_folds,
                       a.scales, a.n_scales, a.walk.stride, a.parts, static_cast<const uint8_t*>(a.state), a.sums);
  };
  if (tiles >= 256) fold(k_adamw_fold<64>, 64);
  else fold(k_adamw_fold<16>, 16);
  return int(hipGetLastError());
}

template <bool kEight>
int convert(const AdamwConvertArgs& a, hipStream_t st) {
  constexpr AdamwShape s = kConvertShape[kEight];
  hipLaunchKernelGGL((k_convert<kEight, s.B, s.U, s.run>), dim3(uint32_t(a.walk.n)), dim3(s.B), s.lds, st, a.from_recs,
                     a.to_recs, a.walk, static_cast<const uint8_t*>(a.from), static_cast<uint8_t*>(a.to), a.seed);
  return int(hipGetLastError());
}

}  // namespace

int launch_adamw_step(const AdamwStepArgs& a, void* stream) {
  const hipStream_t st = hipStream_t(stream);
  if (a.parts) return a.eight ? step<true, true>(a, st) : step<false, true>(a, st);
  return a.eight ? step<true, false>(a, st) : step<false, false>(a, st);
}

int launch_adamw_norm(const AdamwNormArgs& a, void* stream) {
  const hipStream_t st = hipStream_t(stream);
  const uint8_t* grads = static_cast<const uint8_t*>(a.grads);
  const uint32_t n = uint32_t(a.walk.n);
  if (n <= kNormOne) {
    hipLaunchKernelGGL(k_norm<true>, dim3(n ? n : 1), dim3(256), 0, st, a.recs, a.walk, grads, a.max_norm, a.stats,
                       a.parts, a.arrived);
    return int(hipGetLastError());
  }
  hipLaunchKernelGGL(k_norm<false>, dim3(n), dim3(256), 0, st, a.recs, a.walk, grads, a.max_norm, a.stats, a.parts,
                     a.arrived);
  const int e = int(hipGetLastError());
  if (e != 0) return e;
  hipLaunchKernelGGL(k_norm_fold, dim3(kNormFold), dim3(256), 0, st, a.walk.stride, a.walk.n, a.parts,
                     a.parts + 8 * a.walk.stride, a.max_norm, a.stats, a.arrived);
  return int(hipGetLastError());
}

int launch_adamw_scale(float max_norm, fr_grad_stats* stats, void* stream) {
  hipLaunchKernelGGL(k_scale, dim3(1), dim3(1), 0, hipStream_t(stream), max_norm, stats);
  return int(hipGetLastError());
}

int launch_adamw_convert(const AdamwConvertArgs& a, void* stream) {
  return a.eight ? convert<true>(a, hipStream_t(stream)) : convert<false>(a, hipStream_t(stream));
}

}  // namespace fr
