// gfx950 kernels of the step by orthogonalised momentum: the momenta and norms
// of all matrices of a state, the products that orthogonalise them, and the
// step along the updates.
#include <hip/hip_runtime.h>

#include "device.h"
#include "elements.h"
#include "muon.h"

// (momenta and the step are defined operation by operation)
#pragma clang fp contract(off)

namespace fr {
namespace {

typedef _Float16 f16;
typedef f16 f16x4 __attribute__((ext_vector_type(4)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));

// ------------------------------------------------------- walks over elements

struct Elements {
  MuonRec r;
  uint64_t e0;     // the tile's first
  uint32_t n;      // how many it has
  uint32_t place;  // of the tile
};
__device__ __forceinline__ Elements elements_of(const AdamwWalk& w, const MuonRec* recs) {
  Elements t;
  const uint64_t at = (blockIdx.x & 7) * w.stride + (blockIdx.x >> 3);
  const uint64_t slot = w.d[at];
  t.r = recs[slot >> 32];
  t.e0 = uint64_t(uint32_t(slot)) * kMuonTile;
  const uint32_t j = uint32_t(slot), whole = uint32_t(t.r.numel / kMuonTile);
  t.n = j < whole ? kMuonTile : uint32_t(t.r.numel) % kMuonTile;
  t.place = uint32_t(at);
  return t;
}

template <bool kFull>
__device__ __forceinline__ f32x4 load_grad(const void* p, bool f32, uint32_t i, uint32_t n) {
  return __builtin_bit_cast(f32x4, f32 ? load4<kFull>(p, i, n) : widen(load4h<kFull>(p, i, n)));
}

// The tile's sum of x (thread 0's) over its four waves.
template <class T>
__device__ __forceinline__ T tile_sum(T x) {
  __shared__ T part[4];
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = x;
  __syncthreads();
  return part[0] + part[1] + part[2] + part[3];
}

__device__ __forceinline__ float direction(float x, float m, float momentum, bool nesterov) {
  return nesterov ? x + momentum * m : m;
}

// One tile's momenta, the sum of the squares of its directions and, if asked
// for, the momenta's words' sums.
template <bool kMomentum, bool kSums, bool kFull>
__device__ __forceinline__ void momentum_tile(const Elements& t, const MuonArgs& a) {
  const uint32_t n = kFull ? kMuonTile : t.n, i = threadIdx.x * 4;
  const uint8_t* const pg = static_cast<const uint8_t*>(a.grads) + t.r.grad + (t.r.grad_f32 ? 4 : 2) * t.e0;
  f32x4 g = load_grad<kFull>(pg, t.r.grad_f32, i, n), d = g;
  u64 s = 0, ws = 0;
  if constexpr (kMomentum) {
    uint8_t* const pm = static_cast<uint8_t*>(a.state) + t.r.mom + 4 * t.e0;
    u32x4 um = load4<kFull>(pm, i, n);
    const fr_muon_hyper h = a.hyper[t.r.group];
    const fr_grad_stats st = *a.stats;
    if (!st.nonfinite) {
      f32x4 m = __builtin_bit_cast(f32x4, um);
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const float x = g[j] * st.scale;
        m[j] = m[j] * h.momentum + x;
        d[j] = direction(x, m[j], h.momentum, h.nesterov != 0);
        if (!kFull && i + j >= n) m[j] = d[j] = 0.0f;  // (a scale may be NaN)
      }
      um = __builtin_bit_cast(u32x4, m);
      store4<kFull>(pm, um, i, n);
    }
    if constexpr (kSums) acc4(um, uint32_t(4 * t.e0 & (a.C - 1)) / 4 + i, s, ws);
  }
  double q = 0;
#pragma unroll
  for (int j = 0; j < 4; j++) q += double(d[j]) * double(d[j]);
  q = tile_sum(q);
  if (threadIdx.x == 0) a.parts[t.place] = q;
  if constexpr (kSums) {
    s = tile_sum(s);
    __syncthreads();
    ws = tile_sum(ws);
    if (threadIdx.x == 0) a.sum_parts[t.place] = fr_chunk_sum{s, ws};
  }
}

template <bool kMomentum, bool kSums>
__global__ __launch_bounds__(256) void k_muon_momentum(MuonArgs a) {
  const Elements t = elements_of(a.walk, a.recs);
  if (t.n == kMuonTile) momentum_tile<kMomentum, kSums, true>(t, a);
  else momentum_tile<kMomentum, kSums, false>(t, a);
}

// One tile of the step.
template <bool kSums, bool kFull>
__device__ __forceinline__ void apply_tile(const Elements& t, const MuonArgs& a) {
  const uint32_t n = kFull ? kMuonTile : t.n, i = threadIdx.x * 4;
  uint8_t* const pw = static_cast<uint8_t*>(a.state) + t.r.master + 4 * t.e0;
  uint8_t* const pp = t.r.param == kNone ? nullptr : static_cast<uint8_t*>(a.state) + t.r.param + 2 * t.e0;
  u32x4 uw = load4<kFull>(pw, i, n);
  const f32x4 u = __builtin_bit_cast(
      f32x4, widen(load4h<kFull>(static_cast<const uint8_t*>(a.updates) + t.r.update + 2 * t.e0, i, n)));
  const fr_muon_hyper h = a.hyper[t.r.group];
  const bool skip = a.stats->nonfinite != 0;
  u32x2 up = {0, 0};
  if (!skip) {
    const float keep = 1.0f - h.lr * h.weight_decay, step = h.lr * t.r.scale;
    f32x4 w = __builtin_bit_cast(f32x4, uw);
#pragma unroll
    for (int j = 0; j < 4; j++) {
      w[j] = w[j] * keep - u[j] * step;
      if (!kFull && i + j >= n) w[j] = 0.0f;
    }
    uw = __builtin_bit_cast(u32x4, w);
    up = to_bf16(w);
    store4<kFull>(pw, uw, i, n);
    if (pp) store4h<kFull>(pp, up, i, n);
  } else if (kSums && pp) {
    const u32x4 x = widen(load4h<kFull>(pp, i, n));
    up = u32x2{x.x >> 16 | x.y, x.z >> 16 | x.w};
  }
  if constexpr (kSums) {
    u64 s[2] = {}, ws[2] = {};
    acc2(up, uint32_t(2 * t.e0 & (a.C - 1)) / 4 + i / 2, s[0], ws[0]);
    acc4(uw, uint32_t(4 * t.e0 & (a.C - 1)) / 4 + i, s[1], ws[1]);
#pragma unroll
    for (int k = 0; k < 2; k++) {
      s[k] = tile_sum(s[k]);
      __syncthreads();
      ws[k] = tile_sum(ws[k]);
      __syncthreads();
      if (threadIdx.x == 0) a.sum_parts[uint64_t(k) * 8 * a.walk.stride + t.place] = fr_chunk_sum{s[k], ws[k]};
    }
  }
}

template <bool kSums>
__global__ __launch_bounds__(256) void k_muon_apply(MuonArgs a) {
  const Elements t = elements_of(a.walk, a.recs);
  if (t.n == kMuonTile) apply_tile<kSums, true>(t, a);
  else apply_tile<kSums, false>(t, a);
}

// A matrix's norm, and what its elements are multiplied by to be X_0 as it is
// stored.  One workgroup a matrix.
__global__ __launch_bounds__(256) void k_muon_norm(MuonArgs a) {
  const MuonRec& r = a.recs[blockIdx.x];
  double q = 0;
  for (uint64_t i = threadIdx.x; i < r.slots; i += 256) {
    const uint64_t g = r.slot0 + i;
    q += a.parts[(g & 7) * a.walk.stride + (g >> 3)];
  }
  q = tile_sum(q);
  if (threadIdx.x == 0) {
    const double f = double(r.lift) / (__builtin_sqrt(q) + double(a.hyper[r.group].eps));
    a.factors[blockIdx.x] = q == 0.0 ? 0.0 : __builtin_isfinite(q) ? f : __builtin_nan("");
  }
}

// X_0 of a tile: fp32, fp16 and transposed; zeros behind the matrix's sides.
__global__ __launch_bounds__(256) void k_muon_spread(MuonArgs a) {
  if (a.stats->nonfinite) return;
  const uint64_t tile = a.spread.d[blockIdx.x];
  const uint32_t id = uint32_t(tile >> 32), i0 = uint32_t(tile >> 16 & 0xFFFF) * kMuonSide,
                 j0 = uint32_t(tile & 0xFFFF) * kMuonSide;
  const MuonRec r = a.recs[id];
  const double f = a.factors[id];
  const fr_muon_hyper h = a.hyper[r.group];
  const float scale = a.stats->scale;
  const uint8_t* const pg = static_cast<const uint8_t*>(a.grads) + r.grad;
  const float* const pm =
      a.momentum ? reinterpret_cast<const float*>(static_cast<const uint8_t*>(a.state) + r.mom) : nullptr;
  float* const xc = reinterpret_cast<float*>(a.scratch + r.xc);
  f16* const x = reinterpret_cast<f16*>(a.scratch + r.x);
  f16* const xt = reinterpret_cast<f16*>(a.scratch + r.xt[0]);
  __shared__ float t[32][33];
  for (uint32_t q = 0; q < (kMuonSide / 32) * (kMuonSide / 32); q++) {
    const uint32_t bi = i0 + q / (kMuonSide / 32) * 32, bj = j0 + q % (kMuonSide / 32) * 32;
    const uint32_t lo = threadIdx.x % 32, hi = threadIdx.x / 32;
    // read along the matrix's own rows, which are X's or its columns
    for (uint32_t k = hi; k < 32; k += 8) {
      const uint32_t i = r.wide ? bi + k : bi + lo, j = r.wide ? bj + lo : bj + k;
      float d = 0.0f;
      if (i < r.m && j < r.n) {
        const uint64_t e = r.wide ? uint64_t(i) * r.cols + j : uint64_t(j) * r.cols + i;
        d = r.grad_f32 ? reinterpret_cast<const float*>(pg)[e]
                       : as_f(uint32_t(reinterpret_cast<const uint16_t*>(pg)[e]) << 16);
        if (pm) d = direction(d * scale, pm[e], h.momentum, h.nesterov != 0);
        d = float(double(d) * f);
      }
      if (r.wide) t[k][lo] = d;
      else t[lo][k] = d;
    }
    __syncthreads();
    for (uint32_t k = hi; k < 32; k += 8) {
      const uint64_t e = uint64_t(bi + k) * r.np + bj + lo;
      xc[e] = t[k][lo];
      x[e] = f16(t[k][lo]);
      xt[uint64_t(bj + k) * r.mp + bi + lo] = f16(t[lo][k]);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------ products

enum Product { kGram, kPoly, kWhole };

struct ProductArgs {
  const MuonRec* recs;
  const uint64_t* tiles;
  uint8_t* scratch;
  uint8_t* updates;
  const fr_grad_stats* stats;
  float a, b, c;
  uint32_t flip;      // which transpose is read; the other is written
  uint32_t carried;   // X is read as carried, else in fp16
  uint32_t carry;     // and is carried on
  uint32_t last;
};

// One 128 x 128 tile of L R^T, both with their sums' index contiguous: 4 waves of
// 64 x 64, 64 of the sum at a time in LDS, where chunks of 16 bytes are permuted by
// their row so that 16 rows of a column of chunks lie in different banks.
constexpr uint32_t kSide = kMuonSide, kDeep = 64;

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

__device__ __forceinline__ void fetch(const f16* src, uint64_t ld, uint32_t k0, f16* lds) {
  const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x % 64;
#pragma unroll
  for (uint32_t p = 0; p < kSide / 32; p++) {
    const uint32_t row0 = (p * 4 + wave) * 8, row = row0 + lane / 8, chunk = (lane % 8) ^ (row / 2 % 8);
    __builtin_amdgcn_global_load_lds((global_void*)(src + row * ld + k0 + chunk * 8), (lds_void*)(lds + row0 * kDeep),
                                     16, 0, 0);
  }
}

template <Product kWhat>
__global__ __launch_bounds__(256) void k_muon_product(ProductArgs p) {
  if (p.stats->nonfinite) return;
  __shared__ __attribute__((aligned(16))) f16 lds[2][2][kSide * kDeep];
  const uint64_t tile = p.tiles[blockIdx.x];
  const MuonRec r = p.recs[tile >> 32];
  const uint32_t i0 = uint32_t(tile >> 16 & 0xFFFF) * kSide, j0 = uint32_t(tile & 0xFFFF) * kSide;
  f16* const X = reinterpret_cast<f16*>(p.scratch + r.x);
  f16* const A = reinterpret_cast<f16*>(p.scratch + r.a);
  f16* const Q = reinterpret_cast<f16*>(p.scratch + r.q);
  f16* const from = reinterpret_cast<f16*>(p.scratch + (p.flip ? r.xt[1] : r.xt[0]));
  f16* const to = reinterpret_cast<f16*>(p.scratch + (p.flip ? r.xt[0] : r.xt[1]));
  const f16* const L = kWhat == kGram ? X : kWhat == kPoly ? A : Q;
  const f16* const R = kWhat == kGram ? X : kWhat == kPoly ? A : from;
  const uint32_t K = kWhat == kGram ? r.np : r.mp;
  const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x % 64, wi = wave / 2 * 64, wj = wave % 2 * 64;
  const uint32_t row = lane % 16, quad = lane / 16;
  const f16* const pl = L + uint64_t(i0) * K;
  const f16* const pr = R + uint64_t(j0) * K;
  f32x4 acc[4][4] = {};
  fetch(pl, K, 0, lds[0][0]);
  fetch(pr, K, 0, lds[0][1]);
  for (uint32_t k = 0, b = 0; k < K; k += kDeep, b ^= 1) {
    __syncthreads();  // (waits for this wave's loads into LDS as well)
    if (k + kDeep < K) {
      fetch(pl, K, k + kDeep, lds[b ^ 1][0]);
      fetch(pr, K, k + kDeep, lds[b ^ 1][1]);
    }
#pragma unroll
    for (uint32_t kk = 0; kk < 2; kk++) {
      f16x8 x[4], y[4];
#pragma unroll
      for (uint32_t q = 0; q < 4; q++) {
        const uint32_t ri = wi + q * 16 + row, rj = wj + q * 16 + row, ch = kk * 4 + quad;
        x[q] = *reinterpret_cast<const f16x8*>(&lds[b][0][ri * kDeep + (ch ^ (ri / 2 % 8)) * 8]);
        y[q] = *reinterpret_cast<const f16x8*>(&lds[b][1][rj * kDeep + (ch ^ (rj / 2 % 8)) * 8]);
      }
#pragma unroll
      for (uint32_t s = 0; s < 4; s++)
#pragma unroll
        for (uint32_t q = 0; q < 4; q++)
          acc[s][q] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[s], y[q], acc[s][q], 0, 0, 0);
    }
  }
  // a lane holds rows 4 quad ... 4 quad + 3 of column `row` of each 16 x 16
  float* const xc = reinterpret_cast<float*>(p.scratch + r.xc);
#pragma unroll
  for (uint32_t s = 0; s < 4; s++)
#pragma unroll
    for (uint32_t q = 0; q < 4; q++) {
      const uint32_t i = i0 + wi + s * 16 + quad * 4, j = j0 + wj + q * 16 + row;
      f32x4 v = acc[s][q];
      f16x4 h;
      if constexpr (kWhat == kWhole) {
#pragma unroll
        for (uint32_t e = 0; e < 4; e++) {
          const uint64_t at = uint64_t(i + e) * r.np + j;
          const float x = p.carried ? xc[at] : float(X[at]);
          v[e] = __builtin_fmaf(p.a, x, v[e] * (1.0f / kMuonLiftA));
          if (p.carry) xc[at] = v[e];
          h[e] = f16(v[e]);
          if (!p.last) X[at] = h[e];
        }
        if (!p.last) {
          *reinterpret_cast<f16x4*>(to + uint64_t(j) * r.mp + i) = h;
        } else if (j < r.n) {
          uint16_t* const out = reinterpret_cast<uint16_t*>(p.updates + r.update);
          for (uint32_t e = 0; e < 4; e++)
            if (i + e < r.m)
              out[r.wide ? uint64_t(i + e) * r.cols + j : uint64_t(j) * r.cols + i + e] =
                  uint16_t(rne_bf16(as_u(v[e] * (1.0f / r.lift))));
        }
      } else {
        f16* const out = kWhat == kGram ? A : Q;
#pragma unroll
        for (uint32_t e = 0; e < 4; e++) {
          const uint64_t at = uint64_t(i + e) * r.mp + j;
          if constexpr (kWhat == kGram) v[e] *= kMuonLiftA / (r.lift * r.lift);
          else v[e] = __builtin_fmaf(p.b, float(A[at]), p.c * (1.0f / kMuonLiftA) * v[e]);
          h[e] = f16(v[e]);
          out[at] = h[e];
        }
        if (i0 != j0) *reinterpret_cast<f16x4*>(out + uint64_t(j) * r.mp + i) = h;
      }
    }
}

int fold(const MuonArgs& a, hipStream_t st) {
  if (!a.sum_parts || !a.n_folds) return 0;
  AdamwStepArgs f;
  f.walk = a.walk;
  f.folds = a.folds;
  f.n_folds = a.n_folds;
  f.parts = a.sum_parts;
  f.state = a.state;
  f.sums = a.sums;
  return launch_adamw_fold(f, a.C / 2 / kMuonTile, st);
}

}  // namespace

int launch_muon_direction(const MuonArgs& a, void* stream) {
  const hipStream_t st = hipStream_t(stream);
  if (a.walk.n == 0) return 0;
  const dim3 tiles(uint32_t(a.walk.n));
  if (!a.momentum) hipLaunchKernelGGL((k_muon_momentum<false, false>), tiles, dim3(256), 0, st, a);
  else if (a.sum_parts) hipLaunchKernelGGL((k_muon_momentum<true, true>), tiles, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_muon_momentum<true, false>), tiles, dim3(256), 0, st, a);
  if (const int e = int(hipGetLastError())) return e;
  if (const int e = fold(a, st)) return e;
  hipLaunchKernelGGL(k_muon_norm, dim3(a.n), dim3(256), 0, st, a);
  if (const int e = int(hipGetLastError())) return e;
  hipLaunchKernelGGL(k_muon_spread, dim3(uint32_t(a.spread.n)), dim3(256), 0, st, a);
  if (const int e = int(hipGetLastError())) return e;
  for (uint32_t s = 0; s < a.n_steps; s++) {
    ProductArgs p;
    p.recs = a.recs;
    p.scratch = a.scratch;
    p.updates = static_cast<uint8_t*>(a.updates);
    p.stats = a.stats;
    p.a = a.coeffs[s].a;
    p.b = a.coeffs[s].b;
    p.c = a.coeffs[s].c;
    p.flip = s & 1;
    p.last = s + 1 == a.n_steps;
    p.carried = s == 0 || s + 2 < a.n_steps;
    p.carry = s + 3 < a.n_steps;
    p.tiles = a.gram.d;
    hipLaunchKernelGGL(k_muon_product<kGram>, dim3(uint32_t(a.gram.n)), dim3(256), 0, st, p);
    if (const int e = int(hipGetLastError())) return e;
    hipLaunchKernelGGL(k_muon_product<kPoly>, dim3(uint32_t(a.gram.n)), dim3(256), 0, st, p);
    if (const int e = int(hipGetLastError())) return e;
    p.tiles = a.whole.d;
    hipLaunchKernelGGL(k_muon_product<kWhole>, dim3(uint32_t(a.whole.n)), dim3(256), 0, st, p);
    if (const int e = int(hipGetLastError())) return e;
  }
  return 0;
}

int launch_muon_apply(const MuonArgs& a, void* stream) {
  const hipStream_t st = hipStream_t(stream);
  if (a.walk.n == 0) return 0;
  const dim3 tiles(uint32_t(a.walk.n));
  if (a.sum_parts) hipLaunchKernelGGL(k_muon_apply<true>, tiles, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(k_muon_apply<false>, tiles, dim3(256), 0, st, a);
  if (const int e = int(hipGetLastError())) return e;
  return fold(a, st);
}

}  // namespace fr
