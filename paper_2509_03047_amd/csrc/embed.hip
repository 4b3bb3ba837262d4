// gfx950 kernels of the embedding: rows of the state for a batch of tokens, and
// the gradient that they leave.
//
// The gradient's tokens are brought into the order of their rows by one launch:
// each workgroup owns some hundred rows at most, reads all ids (they stay in L2)
// and so counts the tokens of the rows in front of its own as well as its own's,
// by wave; a second pass puts each token at its place.  Its waves have
// consecutive tokens, so the order within a row is the tokens' own, and nothing
// depends on atomics' order.  A row of more than FR_EMBED_RUN tokens is cut into
// runs, which a launch of their own sums up; the last launch writes the rows.
#include <hip/hip_runtime.h>

#include "embed.h"
#include "elements.h"

#pragma clang fp contract(off)

namespace fr {
namespace {

constexpr uint32_t kRun = FR_EMBED_RUN;
constexpr uint32_t kVec = kEmbedVec, kSlice = 64 * kVec;  // columns of a lane, of a wave

// Eight elements from any element's address on (the compiler's own choice of
// loads for what alignment there is).
struct __attribute__((packed, aligned(2))) Half8 {
  uint16_t x[8];
};
struct __attribute__((packed, aligned(4))) Float8 {
  float x[8];
};

struct Cols {
  float x[kVec];
};

// Columns c ... c + 7 of a row of `cols` at p, zeros behind its end.
template <bool kF32>
__device__ __forceinline__ Cols load_cols(const void* p, uint32_t c, uint32_t cols) {
  Cols v;
  if (c + kVec <= cols) {
    if constexpr (kF32) {
      const Float8 f = *reinterpret_cast<const Float8*>(static_cast<const float*>(p) + c);
#pragma unroll
      for (uint32_t j = 0; j < kVec; j++) v.x[j] = f.x[j];
    } else {
      const Half8 h = *reinterpret_cast<const Half8*>(static_cast<const uint16_t*>(p) + c);
#pragma unroll
      for (uint32_t j = 0; j < kVec; j++) v.x[j] = as_f(uint32_t(h.x[j]) << 16);
    }
    return v;
  }
#pragma unroll
  for (uint32_t j = 0; j < kVec; j++) {
    v.x[j] = 0.0f;
    if (c + j < cols)
      v.x[j] = kF32 ? static_cast<const float*>(p)[c + j]
                    : as_f(uint32_t(static_cast<const uint16_t*>(p)[c + j]) << 16);
  }
  return v;
}

template <bool kF32>
__device__ __forceinline__ void store_cols(void* p, const Cols& v, uint32_t c, uint32_t cols) {
  if constexpr (kF32) {
    float* const q = static_cast<float*>(p) + c;
    if (c + kVec <= cols) {
      Float8 f;
#pragma unroll
      for (uint32_t j = 0; j < kVec; j++) f.x[j] = v.x[j];
      *reinterpret_cast<Float8*>(q) = f;
      return;
    }
#pragma unroll
    for (uint32_t j = 0; j < kVec; j++)
      if (c + j < cols) q[j] = v.x[j];
  } else {
    const u32x2 lo = to_bf16(f32x4{v.x[0], v.x[1], v.x[2], v.x[3]}), hi = to_bf16(f32x4{v.x[4], v.x[5], v.x[6], v.x[7]});
    const uint32_t w[4] = {lo.x, lo.y, hi.x, hi.y};
    uint16_t* const q = static_cast<uint16_t*>(p) + c;
    Half8 h;
#pragma unroll
    for (uint32_t j = 0; j < kVec; j++) h.x[j] = uint16_t(w[j / 2] >> (16 * (j & 1)));
    if (c + kVec <= cols) {
      *reinterpret_cast<Half8*>(q) = h;
      return;
    }
#pragma unroll
    for (uint32_t j = 0; j < kVec; j++)
      if (c + j < cols) q[j] = h.x[j];
  }
}

// Token t's row, or `rows` and more if it has none.
__device__ __forceinline__ uint64_t row_at(const EmbedArgs& a, uint64_t t) {
  const int64_t id = a.id_bytes == 4 ? int64_t(static_cast<const int32_t*>(a.ids)[t]) : static_cast<const int64_t*>(a.ids)[t];
  return uint64_t(id) - a.first;
}

// ------------------------------------------------------------------- lookup

template <bool kTable32, bool kOut32>
__global__ __launch_bounds__(256) void k_embed_lookup(EmbedArgs a, uint32_t chunks) {
  const uint64_t g = uint64_t(blockIdx.x) * 256 + threadIdx.x, t = g / chunks;
  if (t >= a.n) return;
  const uint32_t c = uint32_t(g - t * chunks) * kVec;
  const uint64_t row = row_at(a, t);
  Cols v = {};
  if (row < a.rows) {
    v = load_cols<kTable32>(static_cast<const uint8_t*>(a.table) + row * a.cols * (kTable32 ? 4 : 2), c, a.cols);
#pragma unroll
    for (uint32_t j = 0; j < kVec; j++) v.x[j] *= a.scale;
  }
  store_cols<kOut32>(static_cast<uint8_t*>(a.out) + t * a.stride * (kOut32 ? 4 : 2), v, c, a.cols);
}

// ----------------------------------------------------------------- gradient

// Tokens in the order of their rows.  Workgroup g owns rows [g R, (g + 1) R).
__global__ __launch_bounds__(64 * kEmbedWaves) void k_embed_order(EmbedArgs a, uint32_t R) {
  __shared__ uint32_t count[kEmbedWaves][kEmbedRows];  // tokens, then the next place, by wave and row
  __shared__ uint32_t total[64 * kEmbedWaves];
  __shared__ uint32_t below_of[kEmbedWaves];
  const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const uint32_t r0 = blockIdx.x * R, mine = a.rows - r0 < R ? a.rows - r0 : R;
  const uint32_t n = uint32_t(a.n), share = (n + 64 * kEmbedWaves - 1) / (64 * kEmbedWaves) * 64;
  const uint32_t from = wave * share < n ? wave * share : n, to = from + share < n ? from + share : n;
  for (uint32_t i = threadIdx.x; i < kEmbedWaves * kEmbedRows; i += 64 * kEmbedWaves) count[0][i] = 0;
  __syncthreads();
  uint32_t below = 0;
#pragma unroll 4
  for (uint32_t t = from + lane; t < to; t += 64) {
    const uint64_t row = row_at(a, t), in = row - r0;
    if (row < r0) below++;
    else if (in < mine) atomicAdd(&count[wave][in], 1u);
  }
  for (int d = 32; d; d >>= 1) below += __shfl_xor(below, d);
  if (lane == 0) below_of[wave] = below;
  __syncthreads();
  // each row's tokens; then the running sum over rows
  uint32_t own = 0;
  if (threadIdx.x < mine)
    for (uint32_t w = 0; w < kEmbedWaves; w++) own += count[w][threadIdx.x];
  total[threadIdx.x] = own;
  __syncthreads();
  for (uint32_t d = 1; d < kEmbedRows; d *= 2) {
    const uint32_t x = threadIdx.x >= d ? total[threadIdx.x - d] : 0;
    __syncthreads();
    total[threadIdx.x] += x;
    __syncthreads();
  }
  uint32_t base = 0;
  for (uint32_t w = 0; w < kEmbedWaves; w++) base += below_of[w];
  if (threadIdx.x < mine) {
    uint32_t at = base + total[threadIdx.x] - own;
    a.start[r0 + threadIdx.x] = at;
    if (r0 + threadIdx.x + 1 == a.rows) a.start[a.rows] = at + own;
    for (uint32_t w = 0; w < kEmbedWaves; w++) {
      const uint32_t c = count[w][threadIdx.x];
      count[w][threadIdx.x] = at;
      at += c;
    }
  }
  __syncthreads();
  for (uint32_t t0 = from; t0 < to; t0 += 64) {
    const uint32_t t = t0 + lane;
    const uint64_t in = t < to ? row_at(a, t) - r0 : ~uint64_t(0);
    u64 left = __ballot(in < mine);
    while (left) {  // one row of these tokens at a time
      const int leader = __builtin_ctzll(left);
      const uint32_t row = __builtin_amdgcn_readlane(uint32_t(in), leader);
      const u64 same = __ballot(in == row);
      uint32_t at = 0;
      if (int(lane) == leader) at = atomicAdd(&count[wave][row], uint32_t(__builtin_popcountll(same)));
      at = __builtin_amdgcn_readlane(at, leader);
      if (in == row) {
        const uint32_t place = at + uint32_t(__builtin_popcountll(same & ((u64(1) << lane) - 1)));
        a.order[place] = t;
        a.row_of[place] = r0 + row;
      }
      left &= ~same;
    }
  }
}

// Where the sum of the run that starts at place p of a row that starts at s is
// kept.  Of rows with more than kRun tokens one at most starts within kRun places,
// and one at most has a later run that starts there.
__device__ __forceinline__ uint64_t run_slot(uint32_t p, uint32_t s) { return uint64_t(p / kRun) * 2 + (p == s); }

// The sum of `n` <= kRun tokens from place p on.  Four rows are in flight at a
// time; past the end the last one again, not counted.
template <bool kF32>
__device__ __forceinline__ Cols sum_run(const EmbedArgs& a, uint32_t p, uint32_t n, uint32_t c) {
  Cols s = {};
  for (uint32_t i = 0; i < n; i += 4) {
    Cols v[4];
#pragma unroll
    for (uint32_t k = 0; k < 4; k++) {
      const uint32_t t = a.order[p + (i + k < n ? i + k : n - 1)];
      v[k] = load_cols<kF32>(static_cast<const uint8_t*>(a.dout) + uint64_t(t) * a.stride * (kF32 ? 4 : 2), c, a.cols);
    }
#pragma unroll
    for (uint32_t k = 0; k < 4; k++)
      if (i + k < n)
#pragma unroll
        for (uint32_t j = 0; j < kVec; j++) s.x[j] += v[k].x[j];
  }
  return s;
}

// Sums of runs: a wave for each place and slice of columns.
template <bool kF32>
__global__ __launch_bounds__(256) void k_embed_runs(EmbedArgs a, uint32_t slices, uint32_t waves) {
  const uint32_t task = blockIdx.x * 4 + threadIdx.x / 64;
  if (task >= waves) return;
  const uint32_t slot = task / slices, c = (task % slices) * kSlice + threadIdx.x % 64 * kVec;
  const uint32_t all = a.start[a.rows], b = slot / 2 * kRun;  // places b ... b + kRun - 1
  if (b >= all || c >= a.cols) return;
  uint32_t p, e;
  if (slot & 1) {  // of the row that starts here and goes on behind them
    if (b + kRun - 1 >= all) return;
    const uint32_t row = a.row_of[b + kRun - 1];
    p = a.start[row];
    e = a.start[row + 1];
    if (p < b || e - p <= kRun) return;
  } else {  // of the row that has started before
    const uint32_t row = a.row_of[b], s = a.start[row];
    e = a.start[row + 1];
    p = b + s % kRun;
    if (s >= b || e - s <= kRun || p >= e) return;
  }
  const Cols s = sum_run<kF32>(a, p, e - p < kRun ? e - p : kRun, c);
  store_cols<true>(a.runs + uint64_t(slot) * a.cols, s, c, a.cols);
}

// The rows: a wave for each slice of columns of one.
template <bool kF32, bool kGrad32>
__global__ __launch_bounds__(256) void k_embed_rows(EmbedArgs a, uint32_t slices, uint64_t waves) {
  const uint64_t task = uint64_t(blockIdx.x) * 4 + threadIdx.x / 64;
  if (task >= waves) return;
  const uint32_t row = uint32_t(task / slices), c = uint32_t(task % slices) * kSlice + threadIdx.x % 64 * kVec;
  if (c >= a.cols) return;
  const uint32_t s = a.start[row], e = a.start[row + 1], n = e - s;
  if (n == 0 && a.add) return;
  Cols v = {};
  if (n <= kRun) {
    v = sum_run<kF32>(a, s, n, c);
  } else {
    Cols g = {};
    const uint32_t runs = (n + kRun - 1) / kRun;
    for (uint32_t i = 0; i < runs; i++) {
      const Cols x = load_cols<true>(a.runs + run_slot(s + i * kRun, s) * a.cols, c, a.cols);
#pragma unroll
      for (uint32_t j = 0; j < kVec; j++) g.x[j] += x.x[j];
      if (i % kRun == kRun - 1 || i == runs - 1) {
#pragma unroll
        for (uint32_t j = 0; j < kVec; j++) {
          v.x[j] += g.x[j];
          g.x[j] = 0.0f;
        }
      }
    }
  }
#pragma unroll
  for (uint32_t j = 0; j < kVec; j++) v.x[j] *= a.scale;
  uint8_t* const out = static_cast<uint8_t*>(a.grad) + uint64_t(row) * a.cols * (kGrad32 ? 4 : 2);
  if (a.add) {
    const Cols old = load_cols<kGrad32>(out, c, a.cols);
#pragma unroll
    for (uint32_t j = 0; j < kVec; j++) v.x[j] = old.x[j] + v.x[j];
  }
  store_cols<kGrad32>(out, v, c, a.cols);
}

}  // namespace

int launch_embed_lookup(const EmbedArgs& a, void* stream) {
  const hipStream_t st = hipStream_t(stream);
  const uint32_t chunks = (a.cols + kVec - 1) / kVec;
  const uint64_t blocks = (a.n * chunks + 255) / 256;
  if (!blocks) return 0;
  const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(uint32_t(blocks)), dim3(256), 0, st, a, chunks); };
  if (a.table_f32 && a.act_f32) launch(k_embed_lookup<true, true>);
  else if (a.table_f32) launch(k_embed_lookup<true, false>);
  else if (a.act_f32) launch(k_embed_lookup<false, true>);
  else launch(k_embed_lookup<false, false>);
  return int(hipGetLastError());
}

int launch_embed_grad(const EmbedArgs& a, void* stream) {
  const hipStream_t st = hipStream_t(stream);
  if (!a.n && a.add) return 0;
  const uint32_t slices = (a.cols + kSlice - 1) / kSlice;
  const uint32_t R = embed_group_rows(a.rows);
  hipLaunchKernelGGL(k_embed_order, dim3((a.rows + R - 1) / R), dim3(64 * kEmbedWaves), 0, st, a, R);
  if (const int e = int(hipGetLastError())) return e;
  if (a.n > kRun) {
    const uint32_t waves = uint32_t(embed_run_slots(a.n) * slices);
    const auto launch = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((waves + 3) / 4), dim3(256), 0, st, a, slices, waves);
    };
    if (a.act_f32) launch(k_embed_runs<true>);
    else launch(k_embed_runs<false>);
    if (const int e = int(hipGetLastError())) return e;
  }
  const uint64_t waves = uint64_t(a.rows) * slices;
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(uint32_t((waves + 3) / 4)), dim3(256), 0, st, a, slices, waves);
  };
  if (a.act_f32 && a.grad_f32) launch(k_embed_rows<true, true>);
  else if (a.act_f32) launch(k_embed_rows<true, false>);
  else if (a.grad_f32) launch(k_embed_rows<false, true>);
  else launch(k_embed_rows<false, false>);
  return int(hipGetLastError());
}

}  // namespace fr
