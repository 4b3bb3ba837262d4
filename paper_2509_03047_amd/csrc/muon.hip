// gfx950 kernels of the step by orthogonalised momentum: the momenta and norms
// of all matrices of a state, the products that orthogonalise them, and the
// step along the updates.
//
// X <- a X + (b A + c A A) X with A = X X^T is three launches a step over all
// matrices: A, Q = b A + c A A, and a X + Q X.  A and Q are symmetric: of them
// only tiles on and below the diagonal are multiplied, and mirrored.  The smaller
// side is A's (X of a tall matrix is its transpose).
//
// What bounds them, in the share of an 8B model (0.87e9 elements in 224 matrices,
// 22.8 TFLOP, 26.5 ms; a large library product of fp16 reaches 1.3 PFLOP/s here): a
// gram takes 1.38 ms (1.16 PFLOP/s with padding and whole tiles on the diagonal,
// where a library's batch of such products reaches 1.12); a X + Q X 2.9 ms, 0.9, as
// reading and writing X by tiles is not hidden behind the matrix instructions of
// these shorter sums (of 5.7 M cycles 4.0 M are left without it); a square
// product 0.75 to 0.88 ms.  Momenta and norms take 1.45 ms, the step 1.75 (10.5 GB, 6.0
// TB/s) and with sums 1.77: HBM.  X_0 takes 1.53 ms (7.9 GB, 5.1 TB/s): its loads stand
// in branches, so that those of a thread's four parts, the gradient's and the
// momentum's of each, are waited for one after another.  Of eight matrices of 256 x 256 to
// 256 x 1024 a product takes 5 to 9 us and all 122: a chain of launches, whose
// workgroups' loads wait for each other.
#include <hip/hip_runtime.h>

#include <type_traits>

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

// A workgroup takes kMuonTile elements, 4 kMuonSub: each thread four of each sub-tile,
// all of whose loads are in flight together.  A sub-tile lies inside every array's
// chunk.
constexpr uint32_t kU = kMuonTile / kMuonSub;

struct Elements {
  MuonRec r;
  uint64_t e0;     // the tile's first
  uint32_t n;      // how many it has
  uint32_t place;  // of the tile
  uint64_t sub;    // its first sub-tile
};
__device__ __forceinline__ Elements elements_of(const AdamwWalk& w, const MuonRec* recs, uint32_t block) {
  Elements t;
  const uint64_t at = (block & 7) * w.stride + (block >> 3);
  const uint64_t slot = w.d[at];
  t.r = recs[slot >> 32];
  const uint32_t j = uint32_t(slot), whole = uint32_t(t.r.numel / kMuonTile);
  t.e0 = uint64_t(j) * kMuonTile;
  t.n = j < whole ? kMuonTile : uint32_t(t.r.numel) % kMuonTile;
  t.place = uint32_t(at);
  t.sub = t.r.sub0 + uint64_t(j) * kU;
  return t;
}

template <bool kFull>
__device__ __forceinline__ f32x4 load_grad(const void* p, bool f32, uint32_t i, uint32_t n) {
  return __builtin_bit_cast(f32x4, f32 ? load4<kFull>(p, i, n) : widen(load4h<kFull>(p, i, n)));
}

// The sum of x over the workgroup, in all threads.
__device__ __forceinline__ double block_sum(double x) {
  __shared__ double part[4];
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = x;
  __syncthreads();
  return part[0] + part[1] + part[2] + part[3];
}

// A tile's sums: s[u] and ws[u] of its sub-tiles, for `kinds` arrays in turn, added
// up over the workgroup and left where the fold finds them.
__device__ __forceinline__ void leave_sums(const MuonArgs& a, const Elements& t, uint32_t kind, const u64 (&s)[kU],
                                           const u64 (&ws)[kU]) {
  static_assert(kU == 4, "eight values");
  u64 x[8];
#pragma unroll
  for (uint32_t u = 0; u < kU; u++) {
    x[2 * u] = s[u];
    x[2 * u + 1] = ws[u];
  }
  const u64 total = wave_totals(x);
  __shared__ u64 part[2][4][8];
  if (threadIdx.x % 8 == 0) part[kind][threadIdx.x / 64][threadIdx.x % 64 / 8] = total;
  __syncthreads();
  const uint32_t v = threadIdx.x, u = v / 2;
  if (v < 8 && u * kMuonSub < t.n) {
    const uint64_t g = t.sub + u, at = (g & 7) * a.sub_stride + (g >> 3);
    reinterpret_cast<u64*>(a.sum_parts + uint64_t(kind) * 8 * a.sub_stride + at)[v % 2] =
        part[kind][0][v] + part[kind][1][v] + part[kind][2][v] + part[kind][3][v];
  }
}

// Word of sub-tile u's first element in its chunk, by bytes an element.
__device__ __forceinline__ uint32_t word_of(const MuonArgs& a, const Elements& t, uint32_t u, uint32_t bytes) {
  return uint32_t(bytes * (t.e0 + u * kMuonSub) & (a.C - 1)) / 4;
}

__device__ __forceinline__ float direction(float x, float m, float momentum, bool nesterov) {
  return nesterov ? x + momentum * m : m;
}

// One tile's momenta, the sum of the squares of its directions and, if asked
// for, the momenta's words' sums.
template <bool kMomentum, bool kSums, bool kFull>
__device__ __forceinline__ void momentum_tile(const Elements& t, const MuonArgs& a) {
  const uint32_t n = kFull ? kMuonTile : t.n;
  const uint8_t* const pg = static_cast<const uint8_t*>(a.grads) + t.r.grad + (t.r.grad_f32 ? 4 : 2) * t.e0;
  uint8_t* const pm = static_cast<uint8_t*>(a.state) + t.r.mom + 4 * t.e0;
  f32x4 g[kU];
  u32x4 um[kU] = {};
#pragma unroll
  for (uint32_t u = 0; u < kU; u++) {
    const uint32_t i = u * kMuonSub + threadIdx.x * 4;
    if constexpr (kMomentum) um[u] = load4<kFull>(pm, i, n);
    g[u] = load_grad<kFull>(pg, t.r.grad_f32, i, n);
  }
  fr_muon_hyper h = {};
  fr_grad_stats st = {};
  if constexpr (kMomentum) {
    h = a.hyper[t.r.group];
    st = *a.stats;
  }
  double q = 0;
  u64 s[kU] = {}, ws[kU] = {};
#pragma unroll
  for (uint32_t u = 0; u < kU; u++) {
    const uint32_t i = u * kMuonSub + threadIdx.x * 4;
    f32x4 d = g[u];
    if constexpr (kMomentum) {
      if (!st.nonfinite) {
        f32x4 m = __builtin_bit_cast(f32x4, um[u]);
#pragma unroll
        for (int j = 0; j < 4; j++) {
          const float x = g[u][j] * st.scale;
          m[j] = m[j] * h.momentum + x;
          d[j] = direction(x, m[j], h.momentum, h.nesterov != 0);
          if (!kFull && i + j >= n) m[j] = d[j] = 0.0f;  // (a scale may be NaN)
        }
        um[u] = __builtin_bit_cast(u32x4, m);
        store4<kFull>(pm, um[u], i, n);
      }
      if constexpr (kSums) acc4(um[u], word_of(a, t, u, 4) + threadIdx.x * 4, s[u], ws[u]);
    }
#pragma unroll
    for (int j = 0; j < 4; j++) q += double(d[j]) * double(d[j]);
  }
  q = block_sum(q);
  if (threadIdx.x == 0) a.parts[t.place] = q;
  if constexpr (kSums) leave_sums(a, t, 0, s, ws);
}

template <bool kMomentum, bool kSums>
__global__ __launch_bounds__(256) void k_muon_momentum(MuonArgs a) {
  const Elements t = elements_of(a.walk, a.recs, blockIdx.x);
  if (t.n == kMuonTile) momentum_tile<kMomentum, kSums, true>(t, a);
  else momentum_tile<kMomentum, kSums, false>(t, a);
}

// One tile of the step, or with U = 1 (where nothing is summed) one sub-tile: an 8B
// model's share takes 1.75 ms by sub-tiles and 1.80 by tiles, with sums 1.78 by tiles
// and 2.1 by sub-tiles.
template <uint32_t U, bool kFull>
__device__ __forceinline__ void apply_tile(const Elements& t, const MuonArgs& a) {
  constexpr bool kSums = U == kU;
  const uint32_t n = kFull ? U * kMuonSub : t.n;
  uint8_t* const pw = static_cast<uint8_t*>(a.state) + t.r.master + 4 * t.e0;
  uint8_t* const pp = t.r.param == kNone ? nullptr : static_cast<uint8_t*>(a.state) + t.r.param + 2 * t.e0;
  const uint8_t* const pu = static_cast<const uint8_t*>(a.updates) + t.r.update + 2 * t.e0;
  u32x4 uw[U], uu[U];
#pragma unroll
  for (uint32_t k = 0; k < U; k++) {
    const uint32_t i = k * kMuonSub + threadIdx.x * 4;
    uw[k] = load4<kFull>(pw, i, n);
    uu[k] = load4h<kFull>(pu, i, n);
  }
  const fr_muon_hyper h = a.hyper[t.r.group];
  const bool skip = a.stats->nonfinite != 0;
  const float keep = 1.0f - h.lr * h.weight_decay, step = h.lr * t.r.scale;
  u64 s[2][U] = {}, ws[2][U] = {};
#pragma unroll
  for (uint32_t k = 0; k < U; k++) {
    const uint32_t i = k * kMuonSub + threadIdx.x * 4;
    u32x2 up = {0, 0};
    if (!skip) {
      f32x4 w = __builtin_bit_cast(f32x4, uw[k]);
      const f32x4 u = __builtin_bit_cast(f32x4, widen(uu[k]));
#pragma unroll
      for (int j = 0; j < 4; j++) {
        w[j] = w[j] * keep - u[j] * step;
        if (!kFull && i + j >= n) w[j] = 0.0f;
      }
      uw[k] = __builtin_bit_cast(u32x4, w);
      up = to_bf16(w);
      store4<kFull>(pw, uw[k], i, n);
      if (pp) store4h<kFull>(pp, up, i, n);
    } else if (kSums && pp) {
      const u32x4 x = widen(load4h<kFull>(pp, i, n));
      up = u32x2{x.x >> 16 | x.y, x.z >> 16 | x.w};
    }
    if constexpr (kSums) {
      acc2(up, word_of(a, t, k, 2) + threadIdx.x * 2, s[0][k], ws[0][k]);
      acc4(uw[k], word_of(a, t, k, 4) + threadIdx.x * 4, s[1][k], ws[1][k]);
    }
  }
  if constexpr (kSums) {
    leave_sums(a, t, 0, s[0], ws[0]);
    leave_sums(a, t, 1, s[1], ws[1]);
  }
}

template <bool kSums>
__global__ __launch_bounds__(256) void k_muon_apply(MuonArgs a) {
  if constexpr (kSums) {
    const Elements t = elements_of(a.walk, a.recs, blockIdx.x);
    if (t.n == kMuonTile) apply_tile<kU, true>(t, a);
    else apply_tile<kU, false>(t, a);
  } else {
    // sub-tile u of a tile, on the die that the tile belongs to
    const uint32_t u = blockIdx.x / 8 % kU, b = blockIdx.x / (8 * kU) * 8 + blockIdx.x % 8;
    if (b >= a.walk.n) return;
    Elements t = elements_of(a.walk, a.recs, b);
    if (u * kMuonSub >= t.n) return;
    t.e0 += u * kMuonSub;
    t.n = t.n - u * kMuonSub < kMuonSub ? t.n - u * kMuonSub : kMuonSub;
    if (t.n == kMuonSub) apply_tile<1, true>(t, a);
    else apply_tile<1, false>(t, a);
  }
}

// What a matrix's elements are multiplied by to be X_0 as it is stored, from its
// tiles' sums.  A workgroup's 256 threads take turns.
__device__ __forceinline__ double factor_of(const MuonArgs& a, const MuonRec& r) {
  double q = 0;
  for (uint64_t i = threadIdx.x; i < r.slots; i += 256) {
    const uint64_t g = r.slot0 + i;
    q += a.parts[(g & 7) * a.walk.stride + (g >> 3)];
  }
  q = block_sum(q);
  const double f = double(r.lift) / (__builtin_sqrt(q) + double(a.hyper[r.group].eps));
  return q == 0.0 ? 0.0 : __builtin_isfinite(q) ? f : __builtin_nan("");
}

__global__ __launch_bounds__(256) void k_muon_norm(MuonArgs a) {
  const double f = factor_of(a, a.recs[blockIdx.x]);
  if (threadIdx.x == 0) a.factors[blockIdx.x] = f;
}

// ------------------------------------------------------------ X, as carried

// X between steps: fp16, and where the next step wants it closer its rest, in
// steps of 2^-8 of the fp16 number's last place, as 8-bit integers: 19 bits of X in
// all, of elements of any size (below 2^-14, where fp16's steps stay as they are,
// fewer).  Steps multiply directions of small singular values by up to the product of
// their a, 485 times; so where a matrix is of low rank, what X lacks is seen in all
// others: updates of rank 1 are off by 3.3e-3 of their norm with these rests, 4.8e-3
// with four bits (as an e4m3 number has them) and 0.14 without.  As an fp16
// number has 13 bits fewer than its fp32 form, the two add up as integers.
constexpr int kRestShift = 5;

// Four values from their fp16 numbers and the word of their rests, and that word.
__device__ __forceinline__ f32x4 with_rests(const f32x4& h, uint32_t w) {
  f32x4 v;
#pragma unroll
  for (int j = 0; j < 4; j++)
    v[j] = as_f(as_u(h[j]) + (uint32_t(__builtin_amdgcn_sbfe(int(w), 8 * j, 8)) << kRestShift));
  return v;
}
__device__ __forceinline__ uint32_t rests_of(const f32x4& v, const f16x4& h) {
  uint32_t w = 0;
#pragma unroll
  for (int j = 0; j < 4; j++) {  // (of a NaN a NaN's)
    const int more = int(as_u(v[j]) - as_u(float(h[j])) + (1u << (kRestShift - 1))) >> kRestShift;
    w |= uint32_t(uint8_t(more > 127 ? 127 : more < -128 ? -128 : more)) << 8 * j;
  }
  return w;
}

// Four elements from any element's address on, zeros behind the `left` that there are.
template <bool kF32>
__device__ __forceinline__ f32x4 load_four(const void* p, uint64_t at, uint32_t left) {
  f32x4 v = {0, 0, 0, 0};
  if (left >= 4) {
    if constexpr (kF32) {
      v = __builtin_bit_cast(f32x4, u32x4(*reinterpret_cast<const u32x4_at4*>(static_cast<const float*>(p) + at)));
    } else {
      const u32x2 h = *reinterpret_cast<const u32x2_at2*>(static_cast<const uint16_t*>(p) + at);
      v = __builtin_bit_cast(f32x4, u32x4{h.x << 16, h.x & 0xFFFF0000u, h.y << 16, h.y & 0xFFFF0000u});
    }
    return v;
  }
#pragma unroll
  for (uint32_t j = 0; j < 4; j++)
    if (j < left)
      v[j] = kF32 ? static_cast<const float*>(p)[at + j]
                  : as_f(uint32_t(static_cast<const uint16_t*>(p)[at + j]) << 16);
  return v;
}

// X_0 of a tile of 4,096 elements; zeros behind the matrix's sides.  The matrix is
// read along its own rows: 16 of 256 elements where they are X's and there are
// so many, else 64 of 64, by way of LDS where they are X's columns.
template <bool kGrad32>
__device__ __forceinline__ f32x4 spread_four(const MuonArgs& a, const MuonRec& r, const fr_muon_hyper& h, float scale,
                                             double f, uint32_t row, uint32_t col, uint32_t rows) {
  if (row >= rows || col >= r.cols) return f32x4{0, 0, 0, 0};
  const uint64_t at = uint64_t(row) * r.cols + col;
  const uint32_t left = r.cols - col;
  f32x4 d = load_four<kGrad32>(static_cast<const uint8_t*>(a.grads) + r.grad, at, left);
  if (a.momentum) {
    const f32x4 m = load_four<true>(static_cast<const uint8_t*>(a.state) + r.mom, at, left);
#pragma unroll
    for (uint32_t j = 0; j < 4; j++)  // (a scale may be NaN)
      d[j] = j < left ? direction(d[j] * scale, m[j], h.momentum, h.nesterov != 0) : 0.0f;
  }
#pragma unroll
  for (uint32_t j = 0; j < 4; j++) d[j] = j < left ? float(double(d[j]) * f) : 0.0f;
  return d;
}

// kNorms: every workgroup takes its matrix's factor from the tiles' sums itself, a
// launch less, where no matrix has more of them than a workgroup threads.  (With the
// launch and without, us: eight matrices of 64 sums 139.5 and 137.3, of 256 510.7 and
// 508.2; of 1,024 1,043 and 1,052.)
template <bool kNorms>
__global__ __launch_bounds__(256) void k_muon_spread(MuonArgs a) {
  if (a.stats->nonfinite) return;
  const uint64_t tile = a.spread[blockIdx.x];
  const uint32_t id = uint32_t(tile >> 32);
  const MuonRec r = a.recs[id];
  const bool flat = r.wide && r.np % 256 == 0;
  const uint32_t side = flat ? 256 : 64, across = r.np / side;
  const uint32_t i0 = uint32_t(tile) / across * (4096 / side), j0 = uint32_t(tile) % across * side;
  double f;
  if constexpr (kNorms) f = factor_of(a, r);
  else f = a.factors[id];
  const fr_muon_hyper h = a.hyper[r.group];
  const float scale = a.stats->scale;
  f16* const x = reinterpret_cast<f16*>(a.scratch + r.x[0]);
  uint8_t* const rest = a.scratch + r.rest;
  const uint32_t lo = threadIdx.x % (side / 4) * 4, hi = threadIdx.x / (side / 4), down = 1024 / side;
  f32x4 v[4];
#pragma unroll
  for (uint32_t k = 0; k < 4; k++) {
    const uint32_t row = (r.wide ? i0 : j0) + hi + down * k, col = (r.wide ? j0 : i0) + lo;
    v[k] = r.grad_f32 ? spread_four<true>(a, r, h, scale, f, row, col, r.wide ? r.m : r.n)
                      : spread_four<false>(a, r, h, scale, f, row, col, r.wide ? r.m : r.n);
  }
  if (!r.wide) {
    __shared__ float t[64][64 + 1];
#pragma unroll
    for (uint32_t k = 0; k < 4; k++)
#pragma unroll
      for (uint32_t j = 0; j < 4; j++) t[lo + j][hi + 16 * k] = v[k][j];
    __syncthreads();
#pragma unroll
    for (uint32_t k = 0; k < 4; k++)
#pragma unroll
      for (uint32_t j = 0; j < 4; j++) v[k][j] = t[hi + 16 * k][lo + j];
  }
#pragma unroll
  for (uint32_t k = 0; k < 4; k++) {
    const uint64_t at = uint64_t(i0 + hi + down * k) * r.np + j0 + lo;
    const f16x4 y = __builtin_convertvector(v[k], f16x4);
    *reinterpret_cast<f16x4*>(x + at) = y;
    *reinterpret_cast<uint32_t*>(rest + at) = rests_of(v[k], y);
  }
}

// ------------------------------------------------------------------ products

// A = X X^T; polynomials of it from one that is there, or from two; the next X =
// a X + P X.
enum MuonProduct { kGram, kSquare, kPair, kWhole };

// What a launch does.
struct Product {
  // of the square ones, which are read (one by kWhole) and which is written
  uint32_t l, r, out;
  float u, v, w;     // kSquare: u L + w L L; kPair: u L + v R + w L R; kWhole: u X + L X
  uint32_t flip;     // which X is read; the other is written
  uint32_t carried;  // X has a rest
  uint32_t carry;    // and gets one
  uint32_t last;
};
struct ProductArgs {
  const MuonTile* tiles;
  uint32_t n;
  uint8_t* scratch;
  uint8_t* updates;
  const fr_grad_stats* stats;
  Product of[2];  // matrices whose first two steps are taken one by one, and as one
};

// How a workgroup makes a tile of B x B elements: waves of WM x WN, S slices
// of the sum, each D deep, in LDS.
template <uint32_t B_, uint32_t WM_, uint32_t WN_, uint32_t S_>
struct Shape {
  static constexpr uint32_t B = B_, WM = WM_, WN = WN_, S = S_, D = 64;
  static constexpr uint32_t waves = B / WM * (B / WN), threads = 64 * waves;
};
// Large: one workgroup a compute unit (128 KB of slices, 32 of mirrors); a
// wave reads 12 KB of operands for 32 matrix instructions.  (Four waves of 128 x 128
// took 3.3 ms of the share's a X + Q X where eight took 3.03, for copies of sums
// between register files; four or five slices of 32 in turn no less than two of 64.)
// Small: two workgroups a compute unit (72 KB each), four slices for what little there is of
// a sum.
typedef Shape<256, 128, 64, 2> Large;
typedef Shape<64, 32, 32, 4> Small;

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

__device__ __forceinline__ uint32_t lds_address(const f16* p) {
  return uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const f16*)p));
}

// A wave's load into LDS: lane l's 16 bytes from base + offset to `to` + 16 l.  (As
// a builtin it makes the compiler wait for all such loads before each transposing
// read, which it takes to read what they write; arrive() waits for them.  The
// compiler itself has no use for m0 in these kernels, which the tests make sure
// of.)
__device__ __forceinline__ void load_to_lds(const f16* base, uint32_t offset, const f16* to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_address(to)), "v"(offset),
               "s"(base)
               : "memory");
}

// Which column of L R^T a lane of operand R stands for.  Of the 16 columns of a
// matrix instruction's result a lane holds four in turn; those of two are
// interleaved, so that it holds 8 in turn of a row and four lanes 32.
__device__ __forceinline__ uint32_t column_of(uint32_t q, uint32_t lane) {
  return q / 2 * 32 + lane / 4 * 8 + q % 2 * 4 + lane % 4;
}

// A slice of an operand whose rows run along the sum: B rows of D.  Chunks of
// 16 bytes are permuted by their row, so that the 16 rows whose chunk is read at
// one time lie in different banks: rows in turn of L, column_of's of R.
template <bool kR>
__device__ __forceinline__ uint32_t row_key(uint32_t row) {
  return kR ? row / 2 % 2 | row / 8 % 4 * 2 : row / 2 % 8;
}
// (One offset a lane, of the first of a wave's loads: the others' rows have the
// same keys, and the rest of their addresses is a scalar.)
template <class T, bool kR>
struct Rows {
  static constexpr uint32_t kChunks = T::D / 8, kRows = 64 / kChunks;  // of a row, of a wave's load
  uint32_t offset;  // bytes
  __device__ __forceinline__ Rows(uint32_t wave, uint32_t ld) {
    const uint32_t lane = threadIdx.x % 64, row = wave * kRows + lane / kChunks;
    static_assert(T::waves * kRows % 32 == 0, "keys go by rows mod 32");
    offset = (row * ld + ((lane % kChunks) ^ row_key<kR>(row)) * 8) * 2;
  }
  __device__ __forceinline__ void fetch(const f16* src, uint32_t ld, f16* lds, uint32_t wave) const {
#pragma unroll
    for (uint32_t p = 0; p < T::B / kRows / T::waves; p++)
      load_to_lds(src + uint64_t(p * T::waves * kRows) * ld, offset, lds + (p * T::waves + wave) * kRows * T::D);
  }
};
template <class T, bool kR>
__device__ __forceinline__ f16x8 operand_of_row(const f16* lds, uint32_t row, uint32_t chunk) {
  return *reinterpret_cast<const f16x8*>(lds + row * T::D + (chunk ^ row_key<kR>(row)) * 8);
}

// A slice of R where its columns run along the sum: D rows of B.  Chunks are
// permuted so that four columns of four rows each, as read at one time, lie in
// different banks.
template <class T>
__device__ __forceinline__ uint32_t column_key(uint32_t row) {
  return T::B == 64 ? row / 2 % 2 * 4 : row % 4 * 4;
}
template <class T>
struct Columns {
  static constexpr uint32_t kChunks = T::B / 8, kRows = 64 / kChunks;  // of a row, of a wave's load
  uint32_t offset;
  __device__ __forceinline__ Columns(uint32_t wave, uint32_t ld) {
    const uint32_t lane = threadIdx.x % 64, row = wave * kRows + lane / kChunks;
    static_assert(T::waves * kRows % 4 == 0, "keys go by rows mod 4");
    offset = (row * ld + ((lane % kChunks) ^ column_key<T>(row)) * 8) * 2;
  }
  __device__ __forceinline__ void fetch(const f16* src, uint32_t ld, f16* lds, uint32_t wave) const {
#pragma unroll
    for (uint32_t p = 0; p < T::D / kRows / T::waves; p++)
      load_to_lds(src + uint64_t(p * T::waves * kRows) * ld, offset, lds + (p * T::waves + wave) * kRows * T::B);
  }
};
// Rows 32 kk + 8 quad ... + 7 of the lane's column of those from `col` on: a
// transposing read gives a lane four rows of its column for which the 16 lanes
// name four rows of four columns each.
template <class T>
__device__ __forceinline__ f16x8 operand_of_columns(const f16* lds, uint32_t col, uint32_t q, uint32_t kk) {
  const uint32_t lane = threadIdx.x % 64, quad = lane / 16, i = lane % 16;
  const uint32_t c = col + column_of(q, i % 4 * 4);
  union {
    f16x8 v;
    i16x4 half[2];
  } u;
#pragma unroll
  for (uint32_t h = 0; h < 2; h++) {
    const uint32_t k = kk * 32 + quad * 8 + i / 4 + 4 * h;
    u.half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (lds_i16x4*)(lds + k * T::B + ((c / 8) ^ column_key<T>(k)) * 8 + c % 8));
  }
  return u.v;
}

// All of a wave's reads of LDS are done, and all but its last `left` loads into it.
template <uint32_t kLeft>
__device__ __forceinline__ void arrive() {
  static_assert(kLeft < 64, "six bits");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kLeft) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// A wave's operands of 32 of the sum, those in use and those that are read ahead:
// all N of R's, and halves of the M of L's.
template <class T, bool kColumns>
struct Operands {
  static constexpr uint32_t M = T::WM / 16, N = T::WN / 16, H = M / 2;
  static constexpr uint32_t kReadsL = H, kReadsR = kColumns ? 2 * N : N;
  const uint32_t wi, wj;
  f16x8 y[2][N], x[2][H];
  // `kk`: which 32 of the slice
  __device__ __forceinline__ void read_r(uint32_t set, const f16* lds, uint32_t kk) {
    const uint32_t lane = threadIdx.x % 64;
    const f16* const r = lds + T::B * T::D;
#pragma unroll
    for (uint32_t q = 0; q < N; q++)
      y[set][q] = kColumns ? operand_of_columns<T>(r, wj, q, kk)
                           : operand_of_row<T, true>(r, wj + column_of(q, lane % 16), kk * 4 + lane / 16);
  }
  __device__ __forceinline__ void read_l(uint32_t half, const f16* lds, uint32_t kk) {
    const uint32_t lane = threadIdx.x % 64;
#pragma unroll
    for (uint32_t s = 0; s < H; s++)
      x[half][s] = operand_of_row<T, false>(lds, wi + (half * H + s) * 16 + lane % 16, kk * 4 + lane / 16);
  }
  __device__ __forceinline__ void multiply(f32x4 (&acc)[M][N], uint32_t set, uint32_t half) const {
#pragma unroll
    for (uint32_t s = 0; s < H; s++)
#pragma unroll
      for (uint32_t q = 0; q < N; q++)
        acc[half * H + s][q] =
            __builtin_amdgcn_mfma_f32_16x16x32_f16(y[set][q], x[half][s], acc[half * H + s][q], 0, 0, 0);
  }
};

// All of a slice's operands at once, of a wave with few.
template <class T, bool kColumns>
struct SliceOperands {
  static constexpr uint32_t M = T::WM / 16, N = T::WN / 16;
  f16x8 y[T::D / 32][N], x[T::D / 32][M];
  __device__ __forceinline__ void read(const f16* lds, uint32_t wi, uint32_t wj) {
    const uint32_t lane = threadIdx.x % 64;
    const f16* const r = lds + T::B * T::D;
#pragma unroll
    for (uint32_t kk = 0; kk < T::D / 32; kk++) {
#pragma unroll
      for (uint32_t q = 0; q < N; q++)
        y[kk][q] = kColumns ? operand_of_columns<T>(r, wj, q, kk)
                            : operand_of_row<T, true>(r, wj + column_of(q, lane % 16), kk * 4 + lane / 16);
#pragma unroll
      for (uint32_t s = 0; s < M; s++)
        x[kk][s] = operand_of_row<T, false>(lds, wi + s * 16 + lane % 16, kk * 4 + lane / 16);
    }
  }
  __device__ __forceinline__ void multiply(f32x4 (&acc)[M][N]) const {
#pragma unroll
    for (uint32_t kk = 0; kk < T::D / 32; kk++)
#pragma unroll
      for (uint32_t s = 0; s < M; s++)
#pragma unroll
        for (uint32_t q = 0; q < N; q++)
          acc[s][q] = __builtin_amdgcn_mfma_f32_16x16x32_f16(y[kk][q], x[kk][s], acc[s][q], 0, 0, 0);
  }
};

// The order of what stands before it: one of kReads reads of LDS, then its share
// of kProducts matrix instructions.
template <uint32_t kReads, uint32_t kProducts>
__device__ __forceinline__ void interleave() {
  constexpr uint32_t each = kProducts / kReads ? kProducts / kReads : 1;
#pragma unroll
  for (uint32_t i = 0; i < kReads; i++) {
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x008, each, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, kProducts, 0);
  __builtin_amdgcn_sched_barrier(0);
}

// LDS of a workgroup: the ring of slices, and behind it 32 rows of each wave's
// results on their way to the other side of the diagonal.
template <class T>
struct Lds {
  static constexpr uint32_t slice = T::B * T::D;  // of one operand
  static constexpr uint32_t ring = T::S * 2 * slice, mirror = 32 * T::WN;
  static constexpr uint32_t bytes = (ring + T::waves * mirror) * sizeof(f16);
};

// What a workgroup needs to know of a tile to load and multiply.
template <MuonProduct kWhat, class T>
struct Place {
  const MuonRec* rec;
  uint32_t i0, j0, K, ld;  // ld: of R's rows
  const f16 *pl, *pr;
  Rows<T, false> left;
  std::conditional_t<kWhat == kWhole, Columns<T>, Rows<T, true>> right;
  static __device__ __forceinline__ Place of(const ProductArgs& args, uint32_t t, uint32_t wave) {
    const MuonTile& tile = args.tiles[t];
    const MuonRec* const rec = &tile.rec;
    const Product& p = args.of[rec->paired];
    const uint32_t K = kWhat == kGram ? rec->np : rec->mp, ld = kWhat == kWhole ? rec->np : K;
    const f16* const X = reinterpret_cast<const f16*>(args.scratch + rec->x[p.flip]);
    const f16* const L = kWhat == kGram ? X : reinterpret_cast<const f16*>(args.scratch + rec->square[p.l]);
    const f16* const R = kWhat == kPair     ? reinterpret_cast<const f16*>(args.scratch + rec->square[p.r])
                         : kWhat == kSquare ? L
                                            : X;
    const uint32_t i0 = tile.i0, j0 = tile.j0;
    return Place{rec, i0, j0, K, ld, L + uint64_t(i0) * K, kWhat == kWhole ? R + j0 : R + uint64_t(j0) * K,
                 {wave, K}, {wave, ld}};
  }
};

// A wave's way to the other side of the diagonal: 32 rows of its WN columns in 16
// bits, written as they lie and read by columns.  Chunks of 16 bytes are permuted
// by their row; a transposing read gives a lane four rows of its column.  (A
// wave's LDS instructions are carried out in turn.)
template <class T>
struct Mirror {
  static constexpr uint32_t kChunks = T::WN / 8;
  f16* at;
  __device__ __forceinline__ Mirror(f16* lds, uint32_t wave) : at(lds + Lds<T>::ring + wave * Lds<T>::mirror) {}
  // row lane % 16 of the first or second 16, columns 32 c + 8 (lane / 16) ... + 7
  template <class V>
  __device__ __forceinline__ void write(uint32_t half, uint32_t c, const V& v) const {
    static_assert(sizeof(V) == 16, "eight of 16 bits");
    const uint32_t lane = threadIdx.x % 64, row = half * 16 + lane % 16, chunk = c * 4 + lane / 16;
    *reinterpret_cast<V*>(at + row * T::WN + (chunk ^ (row / 2 % kChunks)) * 8) = v;
  }
  // rows 8 (lane / 16) ... + 7 of column 16 q + lane % 16
  __device__ __forceinline__ u32x4 read(uint32_t q) const {
    const uint32_t lane = threadIdx.x % 64, column = q * 16 + lane % 4 * 4;
    union {
      u32x4 v;
      i16x4 half[2];
    } u;
#pragma unroll
    for (uint32_t h = 0; h < 2; h++) {
      const uint32_t k = lane / 16 * 8 + 4 * h + lane % 16 / 4;
      u.half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_i16x4*)(at + k * T::WN + ((column / 8) ^ (k / 2 % kChunks)) * 8 + column % 8));
    }
    return u.v;
  }
};

// What a sum of kSquare or (kTwo) kPair is added to, of two times 16 rows: L and R
// there, and what their diagonals are more.
template <class T, bool kTwo>
struct Terms {
  static constexpr uint32_t N = T::WN / 16;
  f16x8 x[2][N / 2], y[kTwo ? 2 : 1][kTwo ? N / 2 : 1];
  f32x4 ej[N / 2][2];
  float ei[2];
  __device__ __forceinline__ void load(const ProductArgs& args, const MuonRec& rec, const Product& p, uint32_t i,
                                       uint32_t j) {
    const f16* const L = reinterpret_cast<const f16*>(args.scratch + rec.square[p.l]);
    const f16* const R = reinterpret_cast<const f16*>(args.scratch + rec.square[kTwo ? p.r : p.l]);
    const float* const dl = reinterpret_cast<const float*>(args.scratch + rec.diagonal[p.l]);
    const float* const dr = reinterpret_cast<const float*>(args.scratch + rec.diagonal[kTwo ? p.r : p.l]);
#pragma unroll
    for (uint32_t s = 0; s < 2; s++) {
      ei[s] = dl[i + 16 * s];
#pragma unroll
      for (uint32_t c = 0; c < N / 2; c++) {
        x[s][c] = *reinterpret_cast<const f16x8*>(L + uint64_t(i + 16 * s) * rec.mp + j + 32 * c);
        if constexpr (kTwo)
          y[s][c] = *reinterpret_cast<const f16x8*>(R + uint64_t(i + 16 * s) * rec.mp + j + 32 * c);
      }
    }
#pragma unroll
    for (uint32_t c = 0; c < N / 2; c++)
#pragma unroll
      for (uint32_t k = 0; k < 2; k++) ej[c][k] = *reinterpret_cast<const f32x4*>(dr + j + 32 * c + 4 * k);
  }
};

// Tiles of L R (kWhole, with R's columns along the sum) or L R^T, one after
// another: the next one's first slices are loaded while one's results are stored.
template <MuonProduct kWhat, class T>
__global__ __launch_bounds__(T::threads) void k_muon_product(ProductArgs args) {
  const bool skip = args.stats->nonfinite != 0;  // (on its way together with the tile)
  extern __shared__ __attribute__((aligned(16))) f16 lds[];
  constexpr uint32_t kSlice = Lds<T>::slice, M = T::WM / 16, N = T::WN / 16;
  constexpr uint32_t kLoads = 2 * kSlice / (8 * T::threads);  // of a wave, a slice of both operands
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const uint32_t wi = wave / (T::B / T::WN) * T::WM, wj = wave % (T::B / T::WN) * T::WN;
  const Mirror<T> mirror(lds, wave);
  typedef Place<kWhat, T> Here;
  Here here = Here::of(args, blockIdx.x, wave);
  if (skip) return;
  f32x4 acc[M][N];
  typedef Operands<T, kWhat == kWhole> Ops;
  Ops o{wi, wj};
  // Slices lie in a ring: `at` is read, `free` loaded next.
  const f16* at = lds;
  f16* free = lds;
  const auto following = [&](auto* x) { return x == lds + (T::S - 1) * 2 * kSlice ? x - (T::S - 1) * 2 * kSlice : x + 2 * kSlice; };
  const auto fetch = [&](uint32_t k) {
    here.left.fetch(here.pl + k, here.K, free, wave);
    if constexpr (kWhat == kWhole) here.right.fetch(here.pr + uint64_t(k) * here.ld, here.ld, free + kSlice, wave);
    else here.right.fetch(here.pr + k, here.ld, free + kSlice, wave);
    free = following(free);
  };
  const auto fetch_first = [&] {
    at = free = lds;
#pragma unroll
    for (uint32_t s = 0; s < T::S; s++)
      if (s * T::D < here.K) fetch(s * T::D);
  };
  // What is multiplied next is read while something else is.  The first half of
  // 32 of the sum:
  const auto first_half = [&](uint32_t set, uint32_t kk) {
    o.read_l(1, at, kk);
    o.multiply(acc, set, 0);
    interleave<Ops::kReadsL, M * N / 2>();
  };
  // and the second, with what the next 32 begin with.
  const auto second_half = [&](uint32_t set, uint32_t kk) {
    o.read_r(set ^ 1, at, kk);
    o.read_l(0, at, kk);
    o.multiply(acc, set, 1);
    interleave<Ops::kReadsL + Ops::kReadsR, M * N / 2>();
  };
  // A slice, behind which there may be another to load (where there is none, the
  // wait is for all)
  const auto one_slice = [&](uint32_t k, auto more, auto last) {
    first_half(0, 0);
    second_half(0, 1);
    first_half(1, 1);
    if constexpr (last) {
      o.multiply(acc, 1, 1);
    } else {
      // the next slice is there, and nobody reads this one any more
      if constexpr (more) {
        arrive<(T::S - 2) * kLoads>();
        fetch(k + T::S * T::D);
      } else {
        arrive<0>();
      }
      at = following(at);
      second_half(1, 0);
    }
  };
  constexpr std::true_type yes;
  constexpr std::false_type no;

  fetch_first();
  for (uint32_t t = blockIdx.x;;) {
    const Product p = args.of[here.rec->paired];
    // of rows i1 + 16 s a lane holds 8 columns in turn, from j1 + 32 c on
    uint32_t i1 = here.i0 + wi + lane % 16, j1 = here.j0 + wj + lane / 16 * 8;
    // The sums start from what X itself contributes, as far as a product is stored
    // times kMuonLiftA.
    if constexpr (kWhat == kWhole) {
      const f16* const X = reinterpret_cast<const f16*>(args.scratch + here.rec->x[p.flip]);
      // (what L's diagonal is more goes with u)
      const float* const dq = reinterpret_cast<const float*>(args.scratch + here.rec->diagonal[p.l]) + i1;
      float a[M];
#pragma unroll
      for (uint32_t s = 0; s < M; s++) a[s] = p.u * kMuonLiftA + dq[16 * s];
      f16x8 x[M][N / 2];
#pragma unroll
      for (uint32_t s = 0; s < M; s++)
#pragma unroll
        for (uint32_t c = 0; c < N / 2; c++)
          x[s][c] = *reinterpret_cast<const f16x8*>(X + uint64_t(i1 + 16 * s) * here.ld + j1 + 32 * c);
      if (p.carried) {
        const uint8_t* const rest = args.scratch + here.rec->rest;
        u32x2 z[M][N / 2];
#pragma unroll
        for (uint32_t s = 0; s < M; s++)
#pragma unroll
          for (uint32_t c = 0; c < N / 2; c++)
            z[s][c] = *reinterpret_cast<const u32x2*>(rest + uint64_t(i1 + 16 * s) * here.ld + j1 + 32 * c);
#pragma unroll
        for (uint32_t s = 0; s < M; s++)
#pragma unroll
          for (uint32_t q = 0; q < N; q++) {
            // (else its conversions are made before the branch, for both its sides, and take all registers)
            if (q % 2 == 0) asm volatile("" : "+v"(x[s][q / 2]));
            f32x4 v;
#pragma unroll
            for (uint32_t e = 0; e < 4; e++) v[e] = float(x[s][q / 2][q % 2 * 4 + e]);
            acc[s][q] = with_rests(v, z[s][q / 2][q % 2]) * a[s];
          }
      } else {
#pragma unroll
        for (uint32_t s = 0; s < M; s++)
#pragma unroll
          for (uint32_t q = 0; q < N; q++)
#pragma unroll
            for (uint32_t e = 0; e < 4; e++) acc[s][q][e] = a[s] * float(x[s][q / 2][q % 2 * 4 + e]);
      }
    } else {
#pragma unroll
      for (uint32_t s = 0; s < M; s++)
#pragma unroll
        for (uint32_t q = 0; q < N; q++) acc[s][q] = f32x4{0, 0, 0, 0};
    }
    // Of small tiles, what a sum is added to comes before it; large ones have no
    // registers for it.
    constexpr bool kTwo = kWhat == kPair, kAdds = kTwo || kWhat == kSquare, kEarly = kAdds && T::B == kMuonSmall;
    Terms<T, kTwo> early[kEarly ? M / 2 : 1];
    if constexpr (kEarly)
#pragma unroll
      for (uint32_t b = 0; b < M / 2; b++) early[b].load(args, *here.rec, p, i1 + 32 * b, j1);
    const uint32_t K = here.K;
    if (T::S * T::D <= K) arrive<(T::S - 1) * kLoads>();
    else arrive<0>();
    if constexpr (T::B == kMuonSmall) {
      SliceOperands<T, kWhat == kWhole> even, odd;
      even.read(at, wi, wj);
      // the next slice is read while one is multiplied; whether there was one
      const auto slice = [&](uint32_t k, const auto& one, auto& other) {
        const bool next = k + T::D < K;
        if (next) {
          if (k + T::S * T::D <= K) arrive<(T::S - 2) * kLoads>();
          else arrive<0>();
          if (k + T::S * T::D < K) fetch(k + T::S * T::D);
          at = following(at);
          other.read(at, wi, wj);
        }
        one.multiply(acc);
        return next;
      };
      for (uint32_t k = 0; slice(k, even, odd) && slice(k + T::D, odd, even);) k += 2 * T::D;
    } else {
      o.read_r(0, at, 0);
      o.read_l(0, at, 0);
      uint32_t k = 0;
      for (; k + T::S * T::D < K; k += T::D) one_slice(k, yes, no);
      for (; k + T::D < K; k += T::D) one_slice(k, no, no);
      one_slice(k, no, yes);
    }

    const MuonRec* const rec = here.rec;
    const bool diagonal = here.i0 == here.j0;
    const uint32_t i2 = here.j0 + wj + lane % 16, j2 = here.i0 + wi + lane / 16 * 8;  // of the mirror image
    t += gridDim.x;
    const bool more = t < args.n;
    if (more) {
      here = Here::of(args, t, wave);
      arrive<0>();  // nobody reads the ring any more
      fetch_first();
    }
    if constexpr (kWhat == kWhole) {
      const MuonRec& r = *rec;
      f16* const to = reinterpret_cast<f16*>(args.scratch + r.x[p.flip ^ 1]);
      uint8_t* const rest = args.scratch + r.rest;
      const float down = (p.last ? 1.0f / r.lift : 1.0f) / kMuonLiftA;
      // (of a matrix that is tall its rows are X's columns)
      const auto finish_tall = [&] {
        uint16_t* const out = reinterpret_cast<uint16_t*>(args.updates + r.update);
#pragma unroll
        for (uint32_t b = 0; b < M / 2; b++) {
          asm volatile("" ::: "memory");
#pragma unroll
          for (uint32_t s = 2 * b; s < 2 * b + 2; s++)
#pragma unroll
            for (uint32_t c = 0; c < N / 2; c++) {
              const u32x2 lo = to_bf16(acc[s][2 * c] * down), hi = to_bf16(acc[s][2 * c + 1] * down);
              mirror.write(s % 2, c, u32x4{lo.x, lo.y, hi.x, hi.y});
            }
          asm volatile("" ::: "memory");
#pragma unroll
          for (uint32_t q = 0; q < N; q++) {
            const u32x4 v = mirror.read(q);
            const uint32_t row = i2 + q * 16, col = j2 + 32 * b;  // of the matrix
            if (row >= r.n || col >= r.m) continue;
            uint16_t* const to_row = out + uint64_t(row) * r.cols + col;
            if (col + 8 <= r.m) {
              *reinterpret_cast<u32x4_at2*>(to_row) = v;
            } else {
#pragma unroll
              for (uint32_t e = 0; e < 8; e++)
                if (col + e < r.m) to_row[e] = uint16_t(v[e / 2] >> (16 * (e % 2)));
            }
          }
        }
      };
      const auto finish = [&](auto carry, auto last) {
#pragma unroll
        for (uint32_t s = 0; s < M; s++) {
          const uint32_t i = i1 + 16 * s;
#pragma unroll
          for (uint32_t c = 0; c < N / 2; c++) {
            const uint32_t j = j1 + 32 * c;
            const uint64_t to_at = uint64_t(i) * r.np + j;
            const f32x4 v[2] = {acc[s][2 * c] * down, acc[s][2 * c + 1] * down};
            if constexpr (!last) {
              const f16x4 h[2] = {__builtin_convertvector(v[0], f16x4), __builtin_convertvector(v[1], f16x4)};
              *reinterpret_cast<f16x8*>(to + to_at) = __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7);
              if constexpr (carry)
                *reinterpret_cast<u32x2*>(rest + to_at) = u32x2{rests_of(v[0], h[0]), rests_of(v[1], h[1])};
            } else if (i < r.m && j < r.n) {
              uint16_t* const out = reinterpret_cast<uint16_t*>(args.updates + r.update);
              uint16_t* const to_row = out + uint64_t(i) * r.cols + j;
              const u32x2 lo = to_bf16(v[0]), hi = to_bf16(v[1]);
              const u32x4 w = {lo.x, lo.y, hi.x, hi.y};
              if (j + 8 <= r.n) {
                *reinterpret_cast<u32x4_at2*>(to_row) = w;
              } else {
#pragma unroll
                for (uint32_t e = 0; e < 8; e++)
                  if (j + e < r.n) to_row[e] = uint16_t(w[e / 2] >> (16 * (e % 2)));
              }
            }
          }
        }
      };
      if (p.last && !r.wide) finish_tall();
      else if (p.last) finish(no, yes);
      else if (p.carry) finish(yes, no);
      else finish(no, no);
    } else {
      // The rounding of a diagonal, unlike that of other elements, does not average
      // out: what it leaves is kept, and counts in what follows.  With those of L
      // and R, l and r, a product is L R + diag(l) R + L diag(r) of the fp16 ones
      // (but for l r).
      f16* const out = reinterpret_cast<f16*>(args.scratch + rec->square[p.out]);
      float* const left = reinterpret_cast<float*>(args.scratch + rec->diagonal[p.out]);
      const uint32_t ld = rec->mp;
      // Of one operand, the product is symmetric to the last bit; of two, what is on
      // and below the diagonal counts on both sides.
      const bool halves = kTwo && diagonal;
      const float scale = kWhat == kGram ? kMuonLiftA / (rec->lift * rec->lift) : p.w * (1.0f / kMuonLiftA);
#pragma unroll
      for (uint32_t b = 0; b < M / 2; b++) {
        asm volatile("" ::: "memory");
        Terms<T, kTwo> terms;
        if constexpr (kEarly) terms = early[b];
        else if constexpr (kAdds) terms.load(args, *rec, p, i1 + 32 * b, j1);
#pragma unroll
        for (uint32_t s = 2 * b; s < 2 * b + 2; s++)
#pragma unroll
          for (uint32_t c = 0; c < N / 2; c++) {
            const uint32_t i = i1 + 16 * s, j = j1 + 32 * c;
            f16x8 h;
#pragma unroll
            for (uint32_t e = 0; e < 8; e++) {
              float v = scale * acc[s][2 * c + e / 4][e % 4];
              const bool on = diagonal && i == j + e;
              if constexpr (kAdds) {
                const float er = terms.ej[c][e / 4][e % 4], el = terms.ei[s % 2];
                if constexpr (kTwo) {
                  v = __builtin_fmaf(__builtin_fmaf(scale, er, p.u), float(terms.x[s % 2][c][e]), v);
                  v = __builtin_fmaf(__builtin_fmaf(scale, el, p.v), float(terms.y[s % 2][c][e]), v);
                  if (on) v = __builtin_fmaf(p.u, el, __builtin_fmaf(p.v, er, v));
                } else {
                  v = __builtin_fmaf(__builtin_fmaf(scale, el + er, p.u), float(terms.x[s % 2][c][e]), v);
                  if (on) v = __builtin_fmaf(p.u, el, v);
                }
              }
              h[e] = f16(v);
              if (on) left[i] = v - float(h[e]);
            }
            f16* const to = out + uint64_t(i) * ld + j;
            if (!halves || j + 7 <= i) {
              *reinterpret_cast<f16x8*>(to) = h;
            } else {
#pragma unroll
              for (uint32_t e = 0; e < 8; e++)
                if (j + e <= i) to[e] = h[e];
            }
            mirror.write(s % 2, c, h);
          }
        if (diagonal && !halves) continue;
        asm volatile("" ::: "memory");
#pragma unroll
        for (uint32_t q = 0; q < N; q++) {
          const u32x4 h = mirror.read(q);
          const uint32_t i = i2 + q * 16, j = j2 + 32 * b;
          f16* const to = out + uint64_t(i) * ld + j;
          if (!halves || j > i) {
            *reinterpret_cast<u32x4*>(to) = h;
          } else {
#pragma unroll
            for (uint32_t e = 0; e < 8; e++)
              if (j + e > i) reinterpret_cast<uint16_t*>(to)[e] = uint16_t(h[e / 2] >> (16 * (e % 2)));
          }
        }
      }
    }
    if (!more) return;
  }
}

template <class T>
int products(const MuonArgs& a, hipStream_t st) {
  enum { kStep, kPaired, kAll };  // which matrices
  ProductArgs p;
  p.scratch = a.scratch;
  p.updates = static_cast<uint8_t*>(a.updates);
  p.stats = a.stats;
  for (Product& x : p.of) x = Product{};
  const auto launch = [&](auto kernel, const MuonTiles& tiles) {
    p.tiles = tiles.d;
    p.n = uint32_t(tiles.n);
    if (!p.n) return 0;
    const uint32_t grid = T::B == kMuonLarge && p.n > a.units ? a.units : p.n;
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(T::threads), Lds<T>::bytes, st, p);
    return int(hipGetLastError());
  };
  const auto gram = [&](int which) {
    for (Product& x : p.of) x.l = x.r = x.out = 0;
    return launch(k_muon_product<kGram, T>, a.gram[which]);
  };
  const auto pair = [&](int which, uint32_t l, uint32_t r, uint32_t out, float u, float v, float w) {
    for (Product& x : p.of) {
      x.l = l;
      x.r = r;
      x.out = out;
      x.u = u;
      x.v = v;
      x.w = w;
    }
    return l == r ? launch(k_muon_product<kSquare, T>, a.gram[which])
                  : launch(k_muon_product<kPair, T>, a.gram[which]);
  };
  // X goes from step `s` on up to `next`, by u X + L X
  const auto set_whole = [&](Product& x, uint32_t l, float u, uint32_t s, uint32_t next) {
    x.l = l;
    x.u = u;
    x.carried = s == 0 || s + 2 < a.n_steps;
    x.carry = next + 2 < a.n_steps;
    x.last = next == a.n_steps;
  };
  const auto whole = [&](int which) {
    const int e = launch(k_muon_product<kWhole, T>, a.whole[which]);
    for (int i = 0; i < 2; i++) p.of[i].flip ^= which == kAll || which == i;
    return e;
  };
  for (uint32_t s = 0; s < a.n_steps; s++) {
    // (those that have taken the second step with the first have nothing to do in it)
    const int which = s == 1 && a.gram[kPaired].n ? kStep : kAll;
    const fr_muon_coeffs f = a.coeffs[s];
    if (const int e = gram(which)) return e;                             // A
    if (const int e = pair(which, 0, 0, 1, f.b, 0.0f, f.c)) return e;    // Q = b A + c A A
    for (Product& x : p.of) set_whole(x, 1, f.a, s, s + 1);
    if (s == 0 && a.gram[kPaired].n) {
      // Two steps as one, by polynomials of the first A alone: the next A is
      // (a + Q) A (a + Q), and X goes by (a' + Q') (a + Q) = a' a + P.  (No new gram
      // mends errors of A in between, which costs nothing while the singular values
      // are small: of the third and fourth step too, updates would be off by 2.0e-3
      // to 2.9e-3 instead of 1.8e-3.  An 8B share's direction took 26.5 ms instead
      // of 28.5.)
      const fr_muon_coeffs g = a.coeffs[1];
      if (const int e = pair(kPaired, 1, 0, 2, 0.0f, f.a, 1.0f)) return e;  // (a + Q) A
      if (const int e = pair(kPaired, 2, 1, 0, f.a, 0.0f, 1.0f)) return e;  // the next A
      if (const int e = pair(kPaired, 0, 0, 2, g.b, 0.0f, g.c)) return e;   // its Q
      if (const int e = pair(kPaired, 2, 1, 0, f.a, g.a, 1.0f)) return e;   // P
      set_whole(p.of[0], 1, f.a, 0, 1);
      set_whole(p.of[1], 0, f.a * g.a, 0, 2);
    }
    if (const int e = whole(which)) return e;
  }
  return 0;
}

int fold(const MuonArgs& a, hipStream_t st) {
  if (!a.sum_parts || !a.n_folds) return 0;
  AdamwStepArgs f;
  f.walk.stride = a.sub_stride;
  f.folds = a.folds;
  f.n_folds = a.n_folds;
  f.parts = a.sum_parts;
  f.state = a.state;
  f.sums = a.sums;
  return launch_adamw_fold(f, a.C / 2 / kMuonSub, st);
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
  if (a.few_slots) {
    hipLaunchKernelGGL(k_muon_spread<true>, dim3(uint32_t(a.n_spread)), dim3(256), 0, st, a);
  } else {
    hipLaunchKernelGGL(k_muon_norm, dim3(a.n), dim3(256), 0, st, a);
    if (const int e = int(hipGetLastError())) return e;
    hipLaunchKernelGGL(k_muon_spread<false>, dim3(uint32_t(a.n_spread)), dim3(256), 0, st, a);
  }
  if (const int e = int(hipGetLastError())) return e;
  return a.side == kMuonLarge ? products<Large>(a, st) : products<Small>(a, st);
}

int launch_muon_apply(const MuonArgs& a, void* stream) {
  const hipStream_t st = hipStream_t(stream);
  if (a.walk.n == 0) return 0;
  const uint32_t tiles = uint32_t(a.walk.n);
  if (a.sum_parts) hipLaunchKernelGGL(k_muon_apply<true>, dim3(tiles), dim3(256), 0, st, a);
  else hipLaunchKernelGGL(k_muon_apply<false>, dim3((tiles + 7) / 8 * 8 * kU), dim3(256), 0, st, a);
  if (const int e = int(hipGetLastError())) return e;
  return fold(a, st);
}

}  // namespace fr
