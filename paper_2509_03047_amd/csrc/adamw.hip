// gfx950 kernels of the optimizer step: AdamW over all tensors of a state,
// with moments in 32 or 8 bits and, if asked for, the chunk sums of what it
// wrote; the norm of the gradients; moments from one form to the other.
//
// All of them stream: an element's state is read and written once (28 bytes
// with bf16 gradients, 16 with 8-bit moments) for some 20 to 60 instructions,
// so HBM bounds them.  As in the restore's kernels a workgroup takes one tile,
// workgroups follow each other in address order, and a slot table says which
// tile of which tensor each takes.
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

constexpr float kUp = 0x1p112f, kDown = 0x1p-112f;
constexpr int kDrop1 = 20, kDrop2 = 19;  // bits below a code of a first moment, of a root

__device__ __forceinline__ float as_f(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t as_u(float f) { return __builtin_bit_cast(uint32_t, f); }

struct Tile {
  AdamwRec r;
  uint64_t e0;   // its first element
  uint32_t n;    // its elements
  uint32_t place;
};

// The tile of workgroup g.
template <int T>
__device__ __forceinline__ Tile tile_of(const AdamwWalk& w, const AdamwRec* recs, uint64_t g) {
  Tile t;
  const uint64_t at = (g & 7) * w.stride + (g >> 3);
  const uint64_t slot = w.d[at];
  t.r = recs[slot >> 32];
  t.e0 = (slot & 0xFFFFFFFFu) * T;
  const uint64_t left = t.r.numel - t.e0;
  t.n = left < T ? uint32_t(left) : uint32_t(T);
  t.place = uint32_t(at);
  return t;
}

// Elements i ... i + 3 of the n at p, zeros behind them.
__device__ __forceinline__ u32x4 load4(const void* p, uint32_t i, uint32_t n) {
  const uint32_t* q = static_cast<const uint32_t*>(p) + i;
  if (i + 4 <= n) return ld_nt(reinterpret_cast<const u32x4*>(q));
  u32x4 x = {0, 0, 0, 0};
  for (int j = 0; j < 4; j++)
    if (i + j < n) x[j] = q[j];
  return x;
}
// The same of bf16 elements, as fp32 patterns.
__device__ __forceinline__ u32x4 load4h(const void* p, uint32_t i, uint32_t n) {
  const uint16_t* q = static_cast<const uint16_t*>(p) + i;
  if (i + 4 <= n) {
    const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(q));
    return u32x4{x.x << 16, x.x & 0xFFFF0000u, x.y << 16, x.y & 0xFFFF0000u};
  }
  u32x4 x = {0, 0, 0, 0};
  for (int j = 0; j < 4; j++)
    if (i + j < n) x[j] = uint32_t(q[j]) << 16;
  return x;
}
__device__ __forceinline__ void store4(void* p, u32x4 x, uint32_t i, uint32_t n) {
  uint32_t* q = static_cast<uint32_t*>(p) + i;
  if (i + 4 <= n) return st_nt(x, reinterpret_cast<u32x4*>(q));
  for (int j = 0; j < 4; j++)
    if (i + j < n) q[j] = x[j];
}
__device__ __forceinline__ void store4h(void* p, u32x2 x, uint32_t i, uint32_t n) {
  uint16_t* q = static_cast<uint16_t*>(p) + i;
  if (i + 4 <= n) return st_nt2(x, reinterpret_cast<u32x2*>(q));
  for (int j = 0; j < 4; j++)
    if (i + j < n) q[j] = uint16_t(x[j / 2] >> (16 * (j & 1)));
}

// ------------------------------------------------------------ 8-bit moments

__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  for (int d = 32; d; d >>= 1) {
    const uint32_t y = __shfl_xor(x, d);
    x = x > y ? x : y;
  }
  return x;
}

// A block's scale and the factor that its values are encoded with, from the
// pattern of its largest magnitude.
struct Scale {
  float scale, inv;
  bool none;  // every code is 0
};
__device__ __forceinline__ Scale scale_of(uint32_t top) {
  const int e = (int(top - 1) >> 23) + 1;  // of the smallest power of two not below it
  Scale s;
  s.none = e < 28 || e >= 254;
  s.scale = e < 28 ? 0.0f : e >= 254 ? as_f(0x7FC00000u) : as_f(uint32_t(e) << 23);
  s.inv = s.none ? 0.0f : as_f(uint32_t(254 - e) << 23);
  return s;
}
__device__ __forceinline__ uint32_t encode(float x, const Scale& s, uint32_t rnd, int drop) {
  return s.none ? 0 : (as_u(x * s.inv * kDown) + rnd) >> drop;
}
__device__ __forceinline__ float decode1(uint32_t c, float scale) {
  return as_f((c & 127) << kDrop1 | (c & 128) << 24) * kUp * scale;
}
__device__ __forceinline__ float decode2(uint32_t c, float scale) { return as_f(c << kDrop2) * kUp * scale; }

__device__ __forceinline__ uint32_t hash(uint64_t counter, uint32_t seed) {
  uint32_t h = (uint32_t(counter) ^ uint32_t(counter >> 32) * 0x85157AF5u) * 0x9E3779B9u + seed;
  h ^= h >> 16;
  h *= 0xB504F333u;
  h ^= h >> 15;
  h *= 0x93CD3A2Du;
  return h ^ h >> 16;
}

// Codes of four first moments and four roots of second ones, which with those
// of the wave's other lanes make up a block; the block's scales.
__device__ __forceinline__ void encode4(const f32x4& m, const f32x4& r, uint64_t counter, uint32_t seed,
                                        uint32_t* cm, uint32_t* cr, float* sm, float* sr) {
  uint32_t tm = 0, tr = 0;
  for (int j = 0; j < 4; j++) {
    const uint32_t a = as_u(m[j]) & 0x7FFFFFFFu, b = as_u(r[j]) & 0x7FFFFFFFu;
    tm = tm > a ? tm : a;
    tr = tr > b ? tr : b;
  }
  const Scale xm = scale_of(wave_max(tm)), xr = scale_of(wave_max(tr));
  *cm = *cr = 0;
  for (int j = 0; j < 4; j++) {
    uint32_t rm = 1u << (kDrop1 - 1), rr = 1u << (kDrop2 - 1);
    if (seed) {
      const uint32_t h = hash(counter + j, seed);
      rm = h >> 12;
      rr = h & 0x7FFFF;
    }
    const uint32_t a = encode(as_f(as_u(m[j]) & 0x7FFFFFFFu), xm, rm, kDrop1) | (as_u(m[j]) >> 24 & 128);
    *cm |= a << (8 * j);
    *cr |= encode(r[j], xr, rr, kDrop2) << (8 * j);
  }
  *sm = xm.scale;
  *sr = xr.scale;
}

// --------------------------------------------------------------------- step

// The sums of a workgroup's words of K arrays, in thread 0.
template <int K, int B>
__device__ __forceinline__ void block_sums(u64 (&s)[K], u64 (&ws)[K]) {
  __shared__ u64 part[B / 64][2 * K];
  for (int k = 0; k < K; k++)
    for (int d = 32; d; d >>= 1) {
      s[k] += __shfl_xor(s[k], d);
      ws[k] += __shfl_xor(ws[k], d);
    }
  if (threadIdx.x % 64 == 0)
    for (int k = 0; k < K; k++) {
      part[threadIdx.x / 64][k] = s[k];
      part[threadIdx.x / 64][K + k] = ws[k];
    }
  __syncthreads();
  if (threadIdx.x == 0)
    for (int w = 1; w < B / 64; w++)
      for (int k = 0; k < K; k++) {
        s[k] += part[w][k];
        ws[k] += part[w][K + k];
      }
}

template <bool kEight, bool kSums, int B, int U>
__global__ __launch_bounds__(B) void k_adamw(const AdamwRec* recs, AdamwWalk walk, uint8_t* state,
                                             const uint8_t* grads, const fr_adamw_hyper* hyper,
                                             const fr_grad_stats* stats, uint64_t C, fr_chunk_sum* parts) {
  constexpr int K = kEight ? int(kKinds) : int(kKinds32);
  const Tile t = tile_of<B * U * 4>(walk, recs, blockIdx.x);
  const uint32_t n = t.n;
  const bool skip = stats && stats->nonfinite;
  if (skip && !kSums) return;
  uint8_t* const pw = state + t.r.at[kMaster] + 4 * t.e0;
  uint8_t* const pp = t.r.at[kParam] == kNone ? nullptr : state + t.r.at[kParam] + 2 * t.e0;
  uint8_t* const pm = state + t.r.at[kMom1] + (kEight ? 1 : 4) * t.e0;
  uint8_t* const pv = state + t.r.at[kMom2] + (kEight ? 1 : 4) * t.e0;
  float* const psm = kEight ? reinterpret_cast<float*>(state + t.r.at[kScale1]) + t.e0 / FR_ADAMW_BLOCK : nullptr;
  float* const psv = kEight ? reinterpret_cast<float*>(state + t.r.at[kScale2]) + t.e0 / FR_ADAMW_BLOCK : nullptr;
  const uint8_t* const pg = grads + t.r.grad + (t.r.grad_f32 ? 4 : 2) * t.e0;

  const fr_adamw_hyper h = hyper[t.r.group];
  const float gs = stats ? stats->scale : 1.0f;
  const float a1 = 1.0f - h.beta1, a2 = 1.0f - h.beta2;
  const float rb2 = 1.0f / __builtin_sqrtf(h.bias2);
  const float keep = 1.0f - h.lr * h.weight_decay, lr = h.lr / h.bias1;

  u64 s[K] = {}, ws[K] = {};
#pragma unroll
  for (int q = 0; q < U; q++) {
    const uint32_t i = (q * B + threadIdx.x) * 4;
    const bool some = i < n;
    const uint32_t b = i / FR_ADAMW_BLOCK;  // the wave's block
    u32x4 uw = load4(pw, i, n), um, uv;
    u32x2 up = {0, 0};
    uint32_t cm = 0, cv = 0;
    float sm = 0, sv = 0;
    f32x4 m, v;
    if (kEight) {
      if (some) {
        cm = *reinterpret_cast<const uint32_t*>(pm + i);
        cv = *reinterpret_cast<const uint32_t*>(pv + i);
        sm = psm[b];
        sv = psv[b];
      }
      for (int j = 0; j < 4; j++) {
        m[j] = decode1(cm >> (8 * j) & 255, sm);
        v[j] = decode2(cv >> (8 * j) & 255, sv);
        v[j] = v[j] * v[j];
      }
    } else {
      um = load4(pm, i, n);
      uv = load4(pv, i, n);
      m = __builtin_bit_cast(f32x4, um);
      v = __builtin_bit_cast(f32x4, uv);
    }
    if (!skip) {
      const f32x4 g = __builtin_bit_cast(f32x4, t.r.grad_f32 ? load4(pg, i, n) : load4h(pg, i, n));
      f32x4 w = __builtin_bit_cast(f32x4, uw), root;
      for (int j = 0; j < 4; j++) {
        const float x = g[j] * gs;
        m[j] = m[j] * h.beta1 + x * a1;
        v[j] = v[j] * h.beta2 + (x * x) * a2;
        root[j] = __builtin_sqrtf(v[j]);
        const float d = root[j] * rb2 + h.eps;
        w[j] = w[j] * keep - (m[j] / d) * lr;
        if (i + j >= n) m[j] = v[j] = w[j] = root[j] = 0.0f;  // eps may be 0
      }
      uw = __builtin_bit_cast(u32x4, w);
      up = u32x2{rne_bf16(uw.x) | rne_bf16(uw.y) << 16, rne_bf16(uw.z) | rne_bf16(uw.w) << 16};
      store4(pw, uw, i, n);
      if (pp) store4h(pp, up, i, n);
      if (kEight) {
        encode4(m, root, t.r.counter + t.e0 + i, h.seed, &cm, &cv, &sm, &sv);
        if (some) {
          *reinterpret_cast<uint32_t*>(pm + i) = cm;
          *reinterpret_cast<uint32_t*>(pv + i) = cv;
          if (threadIdx.x % 64 == 0) {
            psm[b] = sm;
            psv[b] = sv;
          }
        }
      } else {
        um = __builtin_bit_cast(u32x4, m);
        uv = __builtin_bit_cast(u32x4, v);
        store4(pm, um, i, n);
        store4(pv, uv, i, n);
      }
    } else if (pp) {
      const u32x4 x = load4h(pp, i, n);
      up = u32x2{x.x >> 16 | x.y, x.z >> 16 | x.w};
    }
    if (kSums) {
      const uint64_t e = t.e0 + i, mask = C - 1;
      if (pp) acc2(up, uint32_t(2 * e & mask) / 4, s[kParam], ws[kParam]);
      acc4(uw, uint32_t(4 * e & mask) / 4, s[kMaster], ws[kMaster]);
      if (kEight) {
        const u64 i1 = uint32_t(e & mask) / 4 + 1;
        s[kMom1] += cm;
        ws[kMom1] += i1 * cm;
        s[kMom2] += cv;
        ws[kMom2] += i1 * cv;
        if (some && threadIdx.x % 64 == 0) {
          const u64 is = uint32_t(e / FR_ADAMW_BLOCK * 4 & mask) / 4 + 1;
          s[K - 2] += as_u(sm);
          ws[K - 2] += is * as_u(sm);
          s[K - 1] += as_u(sv);
          ws[K - 1] += is * as_u(sv);
        }
      } else {
        const uint32_t i0 = uint32_t(4 * e & mask) / 4;
        acc4(um, i0, s[kMom1], ws[kMom1]);
        acc4(uv, i0, s[kMom2], ws[kMom2]);
      }
    }
  }
  if (kSums) {
    block_sums<K, B>(s, ws);
    if (threadIdx.x == 0)
      for (int k = 0; k < K; k++) parts[uint64_t(t.place) * K + k] = fr_chunk_sum{s[k], ws[k]};
  }
}

// A chunk's sums from what its tiles left: 16 lanes a chunk.
template <int K>
__global__ __launch_bounds__(256) void k_adamw_fold(const AdamwFold* folds, uint32_t n_folds, uint64_t stride,
                                                    const fr_chunk_sum* parts, fr_chunk_sum* sums) {
  const uint32_t f = (blockIdx.x * 256 + threadIdx.x) / 16, lane = threadIdx.x % 16;
  u64 s = 0, ws = 0;
  AdamwFold d = {};
  if (f < n_folds) {
    d = folds[f];
    for (uint32_t j = lane; j < d.n; j += 16) {
      const uint64_t g = uint64_t(d.slot) + j;
      const fr_chunk_sum x = parts[((g & 7) * stride + (g >> 3)) * K + d.kind];
      s += x.sum;
      ws += x.wsum;
    }
  }
  for (int x = 8; x; x >>= 1) {
    s += __shfl_xor(s, x);
    ws += __shfl_xor(ws, x);
  }
  if (f < n_folds && lane == 0) sums[d.chunk] = fr_chunk_sum{s, ws};
}

// --------------------------------------------------------------------- norm

__device__ __forceinline__ void set_stats(double sum_sq, float max_norm, fr_grad_stats* out) {
  const bool fine = __builtin_isfinite(sum_sq);
  const float norm = float(__builtin_sqrt(sum_sq));
  out->sum_sq = sum_sq;
  out->norm = norm;
  out->scale = !fine ? 0.0f : norm > max_norm ? max_norm / norm : 1.0f;
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

// Workgroup g takes tiles g, g + G, ...; the one that ends last adds up what
// all have left, each thread and the whole in an order of their own, whoever
// it is.
__global__ __launch_bounds__(256) void k_norm(const AdamwRec* recs, AdamwWalk walk, const uint8_t* grads,
                                              float max_norm, fr_grad_stats* stats, double* parts,
                                              uint32_t* arrived) {
  double sum = 0;
  for (uint64_t g = blockIdx.x; g < walk.n; g += gridDim.x) {
    const Tile t = tile_of<kNormTile>(walk, recs, g);
    const uint8_t* const p = grads + t.r.grad + (t.r.grad_f32 ? 4 : 2) * t.e0;
    for (uint32_t i = threadIdx.x * 4; i < t.n; i += 256 * 4) {
      const f32x4 x = __builtin_bit_cast(f32x4, t.r.grad_f32 ? load4(p, i, t.n) : load4h(p, i, t.n));
      for (int j = 0; j < 4; j++) sum += double(x[j]) * double(x[j]);
    }
  }
  sum = block_sum(sum);
  __shared__ bool last;
  if (threadIdx.x == 0) {
    __hip_atomic_store(parts + blockIdx.x, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    last = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  sum = 0;
  for (uint32_t i = threadIdx.x; i < gridDim.x; i += 256)
    sum += __hip_atomic_load(parts + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  sum = block_sum(sum);
  if (threadIdx.x == 0) {
    set_stats(sum, max_norm, stats);
    __hip_atomic_store(arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

__global__ void k_scale(float max_norm, fr_grad_stats* stats) { set_stats(stats->sum_sq, max_norm, stats); }

// ------------------------------------------------------------------ convert

template <bool kEight, int B, int U>
__global__ __launch_bounds__(B) void k_convert(const AdamwRec* from_recs, const AdamwRec* to_recs, AdamwWalk walk,
                                               const uint8_t* from, uint8_t* to, uint32_t seed) {
  const Tile t = tile_of<B * U * 4>(walk, to_recs, blockIdx.x);
  const AdamwRec f = from_recs[walk.d[t.place] >> 32];
  const bool f8 = f.at[kScale1] != kNone;
  const uint64_t b0 = t.e0 / FR_ADAMW_BLOCK;
  const uint8_t* const qm = from + f.at[kMom1] + (f8 ? 1 : 4) * t.e0;
  const uint8_t* const qv = from + f.at[kMom2] + (f8 ? 1 : 4) * t.e0;
  const float* const qsm = f8 ? reinterpret_cast<const float*>(from + f.at[kScale1]) + b0 : nullptr;
  const float* const qsv = f8 ? reinterpret_cast<const float*>(from + f.at[kScale2]) + b0 : nullptr;
  uint8_t* const pm = to + t.r.at[kMom1] + (kEight ? 1 : 4) * t.e0;
  uint8_t* const pv = to + t.r.at[kMom2] + (kEight ? 1 : 4) * t.e0;
  float* const psm = kEight ? reinterpret_cast<float*>(to + t.r.at[kScale1]) + b0 : nullptr;
  float* const psv = kEight ? reinterpret_cast<float*>(to + t.r.at[kScale2]) + b0 : nullptr;
#pragma unroll
  for (int q = 0; q < U; q++) {
    const uint32_t i = (q * B + threadIdx.x) * 4;
    const bool some = i < t.n;
    const uint32_t b = i / FR_ADAMW_BLOCK;
    f32x4 m = {0, 0, 0, 0}, v = m;
    uint32_t cm = 0, cv = 0;
    float sm = 0, sv = 0;
    if (f8) {
      if (some) {
        cm = *reinterpret_cast<const uint32_t*>(qm + i);
        cv = *reinterpret_cast<const uint32_t*>(qv + i);
        sm = qsm[b];
        sv = qsv[b];
      }
      if (!kEight)
        for (int j = 0; j < 4; j++) {
          m[j] = decode1(cm >> (8 * j) & 255, sm);
          v[j] = decode2(cv >> (8 * j) & 255, sv);
          v[j] = v[j] * v[j];
        }
    } else {
      m = __builtin_bit_cast(f32x4, load4(qm, i, t.n));
      v = __builtin_bit_cast(f32x4, load4(qv, i, t.n));
      if (kEight) {
        for (int j = 0; j < 4; j++) v[j] = __builtin_sqrtf(v[j]);
        encode4(m, v, t.r.counter + t.e0 + i, seed, &cm, &cv, &sm, &sv);
      }
    }
    if (kEight) {
      if (some) {
        *reinterpret_cast<uint32_t*>(pm + i) = cm;
        *reinterpret_cast<uint32_t*>(pv + i) = cv;
        if (threadIdx.x % 64 == 0) {
          psm[b] = sm;
          psv[b] = sv;
        }
      }
    } else {
      store4(pm, __builtin_bit_cast(u32x4, m), i, t.n);
      store4(pv, __builtin_bit_cast(u32x4, v), i, t.n);
    }
  }
}

template <bool kEight, bool kSums, int B, int U>
int step(const AdamwStepArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((k_adamw<kEight, kSums, B, U>), dim3(uint32_t(a.walk.n)), dim3(B), 0, st, a.recs, a.walk,
                     static_cast<uint8_t*>(a.state), static_cast<const uint8_t*>(a.grads), a.hyper, a.stats, a.C,
                     a.parts);
  return int(hipGetLastError());
}

template <bool kEight>
int step_of(const AdamwStepArgs& a, hipStream_t st) {
  if (!a.parts) return step<kEight, false, 256, kStepTile / 1024>(a, st);
  const int e = a.tile == kStepTile ? step<kEight, true, 256, kStepTile / 1024>(a, st)
                                    : step<kEight, true, 256, kSmallTile / 1024>(a, st);
  if (e != 0 || a.n_folds == 0) return e;
  constexpr int K = kEight ? int(kKinds) : int(kKinds32);
  hipLaunchKernelGGL((k_adamw_fold<K>), dim3((a.n_folds + 15) / 16), dim3(256), 0, st, a.folds, a.n_folds,
                     a.walk.stride, a.parts, a.sums);
  return int(hipGetLastError());
}

}  // namespace

int launch_adamw_step(const AdamwStepArgs& a, void* stream) {
  return a.eight ? step_of<true>(a, hipStream_t(stream)) : step_of<false>(a, hipStream_t(stream));
}

int launch_adamw_norm(const AdamwNormArgs& a, void* stream) {
  const uint32_t groups = a.walk.n < 1 ? 1 : a.walk.n < kNormGroups ? uint32_t(a.walk.n) : kNormGroups;
  hipLaunchKernelGGL(k_norm, dim3(groups), dim3(256), 0, hipStream_t(stream), a.recs, a.walk,
                     static_cast<const uint8_t*>(a.grads), a.max_norm, a.stats, a.parts, a.arrived);
  return int(hipGetLastError());
}

int launch_adamw_scale(float max_norm, fr_grad_stats* stats, void* stream) {
  hipLaunchKernelGGL(k_scale, dim3(1), dim3(1), 0, hipStream_t(stream), max_norm, stats);
  return int(hipGetLastError());
}

int launch_adamw_convert(const AdamwConvertArgs& a, void* stream) {
  const dim3 grid(uint32_t(a.walk.n)), block(256);
  const hipStream_t st = hipStream_t(stream);
  const uint8_t* from = static_cast<const uint8_t*>(a.from);
  uint8_t* to = static_cast<uint8_t*>(a.to);
  if (a.eight)
    hipLaunchKernelGGL((k_convert<true, 256, kStepTile / 1024>), grid, block, 0, st, a.from_recs, a.to_recs, a.walk,
                       from, to, a.seed);
  else
    hipLaunchKernelGGL((k_convert<false, 256, kStepTile / 1024>), grid, block, 0, st, a.from_recs, a.to_recs, a.walk,
                       from, to, a.seed);
  return int(hipGetLastError());
}

}  // namespace fr
